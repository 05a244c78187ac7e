"""Operators around the training step, without a GPU: what the entry points refuse before anything is launched, and the
oracle that the GPU tests compare with (gradients against differences, formats against torch's, rounding without bias)."""
import ctypes
import os
import types

import numpy as np
import pytest
import torch

from oracle import operators_oracle as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, ODD = 1 << 20, (1 << 20) + 4      # an aligned and a misaligned address; every call below is refused before it is used


@pytest.fixture(scope="module")
def K():
    import __graft_entry__ as g
    if not os.path.exists(os.path.join(ROOT, "paper_2603_21014_amd", "libclt.so")):
        g.build()
    from paper_2603_21014_amd import binding
    return binding


def refused(K, code, word, rc):
    assert rc == code, (rc, K._lib.clt_last_error(None))
    assert word in K._lib.clt_last_error(None).decode()


def test_rms_norm_refusals(K):
    f = K._lib.clt_rms_norm

    def call(L=2, B=3, d=64, dtype=K.DTYPE_BF16, x=P, residual=None, weight=P, eps=1e-5, h=None, y=P, q=None, q_scale=None, rstd=None):
        return f(None, L, B, d, dtype, x, residual, weight, eps, h, y, q, q_scale, rstd)
    for bad in (dict(L=0), dict(L=129), dict(B=0), dict(B=-1), dict(d=0), dict(d=12), dict(d=(1 << 20) + 8), dict(L=128, B=1 << 24)):
        refused(K, -2, "shape", call(**bad))
    refused(K, -1, "dtype", call(dtype=2))
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        refused(K, -1, "eps", call(eps=eps))
    refused(K, -1, "argument x is NULL", call(x=None))
    refused(K, -1, "weight is NULL", call(weight=None))
    refused(K, -1, "go together", call(residual=P))
    refused(K, -1, "go together", call(h=P))
    refused(K, -1, "go together", call(q=P))
    refused(K, -1, "go together", call(q_scale=P))
    refused(K, -1, "neither", call(y=None))
    for name in ("x", "weight", "y", "rstd"):
        refused(K, -3, name, call(**{name: ODD}))
    refused(K, -3, "q_scale", call(q=P, q_scale=ODD))
    refused(K, -3, "argument h", call(residual=P, h=ODD))


def test_rms_norm_backward_refusals(K):
    n = K.clt_rms_norm_backward_workspace_bytes(2, 300, 64)
    assert n > 0 and n % 4 == 0
    assert K._lib.clt_rms_norm_backward_workspace_bytes(2, 300, 64, None) == -1
    with pytest.raises(K.CLTError) as e:
        K.clt_rms_norm_backward_workspace_bytes(2, 300, 63)
    assert e.value.code == -2

    def call(L=2, B=300, d=64, dtype=K.DTYPE_F32, h=P, weight=P, rstd=P, dy=P, dh=None, dx=P, dweight=P, ws=P, nbytes=n):
        return K._lib.clt_rms_norm_backward(None, L, B, d, dtype, h, weight, rstd, dy, dh, dx, dweight, ws, nbytes)
    refused(K, -2, "shape", call(d=4))
    refused(K, -1, "dtype", call(dtype=-1))
    for name in ("h", "weight", "rstd", "dy", "dx"):
        refused(K, -1, f"argument {name} is NULL", call(**{name: None}))
        refused(K, -3, f"argument {name}", call(**{name: ODD}))
    refused(K, -3, "argument dh", call(dh=ODD))
    for bad in (dict(ws=None), dict(ws=ODD), dict(nbytes=n - 1)):
        refused(K, -4, "workspace", call(**bad))


def test_adamw_refusals(K):
    assert ctypes.sizeof(K.clt_adamw_tensor) == 7 * 8 + 8 + 4 * 4

    def tensor(p=P, g=P, m=P, v=P, m_scale=None, v_scale=None, master=None, n=100, dtype=0, grad_dtype=0, bits=32, decay=0.0):
        return K.clt_adamw_tensor(p, g, m, v, m_scale, v_scale, master, n, dtype, grad_dtype, bits, decay)

    def call(*tensors, count=None, t=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8):
        a = (K.clt_adamw_tensor * max(1, len(tensors)))(*tensors)
        return K._lib.clt_adamw_step(None, len(tensors) if count is None else count, a, t, lr, b1, b2, eps, 0)
    good8 = dict(m_scale=P, v_scale=P, bits=8)
    refused(K, -1, "list", call(count=-1))
    assert K._lib.clt_adamw_step(None, 1, None, 1, 1e-3, 0.9, 0.999, 1e-8, 0) == -1
    refused(K, -1, "step count", call(tensor(), t=0))
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(eps=float("inf")), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(eps=0.0), dict(eps=1e-60), dict(eps=1e-39)):
        refused(K, -1, "scalar", call(tensor(), **bad))
    refused(K, -2, "tensor 1", call(tensor(**good8), tensor(n=-1)))
    refused(K, -2, "tensor 0", call(tensor(n=(1 << 34) + 1)))
    for bad in (dict(dtype=2), dict(grad_dtype=2), dict(bits=16), dict(decay=-0.1), dict(decay=float("nan")), dict(decay=float("inf"))):
        refused(K, -1, "tensor 1", call(tensor(), tensor(**bad)))
    for name in ("p", "g", "m", "v"):
        refused(K, -1, "required", call(tensor(**{name: None})))
        refused(K, -3, "aligned", call(tensor(**{name: ODD})))
    refused(K, -1, "8-bit", call(tensor(bits=8)))
    refused(K, -1, "8-bit", call(tensor(bits=8, m_scale=P)))
    refused(K, -1, "8-bit", call(tensor(m_scale=P, v_scale=P)))
    refused(K, -3, "aligned", call(tensor(**dict(good8, v_scale=ODD))))
    refused(K, -3, "aligned", call(tensor(master=ODD)))
    # nothing to do is no error, and needs no device
    assert call(count=0) == 0 and call(tensor(n=0, p=None, g=None, m=None, v=None)) == 0


def test_adamw_scalars_that_are_infinite_in_32_bits_are_refused(K):
    """Finite doubles whose rounding, or quotient with the bias correction, is no finite float: an element without a gradient would be NaN."""
    def call(lr=1e-3, b1=0.9, decay=0.0, n=100, t=1):
        a = (K.clt_adamw_tensor * 1)(K.clt_adamw_tensor(P, P, P, P, None, None, None, n, 0, 0, 32, decay))
        return K._lib.clt_adamw_step(None, 1, a, t, lr, b1, 0.999, 1e-8, 0)
    for bad in (dict(lr=1e39), dict(lr=1e300), dict(lr=1e38, b1=0.99), dict(lr=1e308, b1=0.999, n=0)):
        refused(K, -1, "scalar", call(**bad))
    refused(K, -1, "weight_decay", call(lr=1e10, decay=1e30))
    for good in (dict(lr=1e38, b1=0.0, n=0), dict(lr=1e37, t=10 ** 6, n=0)):
        assert call(**good) == 0


def test_outputs_that_overlap_are_refused(K):
    at = lambda k: (k + 1) << 24      # places 16 MB apart
    L, B, d = 2, 3, 64
    n = L * B * d * 2

    def norm(**kw):
        a = dict(x=at(0), residual=at(1), weight=at(2), h=at(3), y=at(4), q=at(5), q_scale=at(6), rstd=at(7))
        a.update(kw)
        return K._lib.clt_rms_norm(None, L, B, d, K.DTYPE_BF16, a["x"], a["residual"], a["weight"], 1e-5, a["h"], a["y"], a["q"], a["q_scale"], a["rstd"])
    for kw in (dict(y=at(0)), dict(y=at(1) + n - 16), dict(y=at(3)), dict(q=at(0) + 16), dict(q=at(4)), dict(q_scale=at(2)), dict(rstd=at(6)), dict(h=at(0) + 16), dict(h=at(1) - 16),
               dict(h=at(2)), dict(h=at(0), y=at(0))):
        refused(K, -1, "overlaps", norm(**kw))

    def back(**kw):
        a = dict(h=at(0), weight=at(1), rstd=at(2), dy=at(3), dh=at(4), dx=at(5), dweight=at(6), ws=at(7))
        a.update(kw)
        return K._lib.clt_rms_norm_backward(None, L, B, d, K.DTYPE_BF16, a["h"], a["weight"], a["rstd"], a["dy"], a["dh"], a["dx"], a["dweight"], a["ws"], 1 << 20)
    for kw in (dict(dx=at(0)), dict(dx=at(3) + 16), dict(dx=at(4) - 16), dict(dweight=at(1)), dict(dweight=at(5)), dict(ws=at(0)), dict(ws=at(6) - 16), dict(dx=at(2))):
        refused(K, -1, "overlaps", back(**kw))
    rows, Kd = 24, 64
    for a, s, c, sc in ((at(0), None, at(0), at(2)), (at(0), None, at(1), at(1) + 4096), (at(0), None, at(1), at(0) + 16)):
        refused(K, -1, "overlaps", K._lib.clt_mx4_quantise(None, L, rows, Kd, K.DTYPE_BF16, K.INPUT_NATIVE, 0, a, s, c, sc))
    refused(K, -1, "overlaps", K._lib.clt_mx4_quantise(None, L, rows, Kd, K.DTYPE_BF16, K.INPUT_INT8_ROWSCALE, 0, at(0), at(1), at(2), at(1)))
    for c, s, o in ((at(0), at(1), at(0) + 4096), (at(0), at(1), at(1))):
        refused(K, -1, "overlaps", K._lib.clt_mx4_dequantise(None, L, rows, Kd, 1, c, s, o))
    for k in range(6):
        args = [at(i) for i in range(6)]
        refused(K, -1, "overlaps", K._lib.clt_mx4_product(None, L, 5, 24, Kd, *args, 0, args[k] + 16))


def test_norm_in_place_keeps_its_other_inputs_apart(K):
    """The sum may overwrite x or residual, but not a part of the other one or the weights under it."""
    at = lambda k: (k + 1) << 24
    n = 2 * 3 * 64 * 2

    def norm(x, residual, weight, h):
        return K._lib.clt_rms_norm(None, 2, 3, 64, K.DTYPE_BF16, x, residual, weight, 1e-5, h, at(7), None, None, None)
    for a, b in ((at(0), at(0) + 128), (at(0), at(0) - 128), (at(0), at(0) + n - 16), (at(0) + 16, at(0))):
        refused(K, -1, "overlaps", norm(a, b, at(2), a))
        refused(K, -1, "overlaps", norm(a, b, at(2), b))
    for w in (at(0), at(0) + n - 16, at(0) - 2 * 64 * 4 + 16):
        refused(K, -1, "overlaps", norm(at(0), at(1), w, at(0)))
        refused(K, -1, "overlaps", norm(at(1), at(0), w, at(0)))
    # one buffer as both operands holds twice itself afterwards, and neighbours are no overlap: these get as far as the device
    for args in ((at(0), at(0), at(2), at(0)), (at(0), at(0) + n, at(2), at(0)), (at(0), at(1), at(0) + n, at(0))):
        if not torch.cuda.is_available():
            assert norm(*args) == -5, K._lib.clt_last_error(None)


def test_mx4_refusals(K):
    assert K.clt_mx4_bytes(3, 65, 136) == (3 * 2 * 2 * 4096, 3 * 2 * 2 * 256)
    for bad in ((0, 8, 64), (1, 0, 64), (1, 8, 0), (1, 8, 12), (65536, 8, 64), (1, (1 << 20) + 1, 64), (1, 1 << 20, 1 << 16), (1, 8, (1 << 22) + 8)):
        with pytest.raises(K.CLTError) as e:
            K.clt_mx4_bytes(*bad)
        assert e.value.code == -2
    assert K._lib.clt_mx4_bytes(1, 8, 64, None, None) == -1

    def quantise(L=2, rows=24, K_=64, dtype=K.DTYPE_BF16, fmt=K.INPUT_NATIVE, transposed=0, a=P, a_scale=None, codes=P, scales=P):
        return K._lib.clt_mx4_quantise(None, L, rows, K_, dtype, fmt, transposed, a, a_scale, codes, scales)
    i8 = K.INPUT_INT8_ROWSCALE
    refused(K, -2, "shape", quantise(K_=60))
    refused(K, -2, "multiple of 8", quantise(rows=20, transposed=1))
    for bad in (dict(dtype=2), dict(fmt=2), dict(transposed=2), dict(fmt=i8, dtype=K.DTYPE_F32, a_scale=P)):
        refused(K, -1, "bad dtype", quantise(**bad))
    refused(K, -1, "transposed", quantise(fmt=i8, a_scale=P, transposed=1))
    refused(K, -1, "a_scale", quantise(fmt=i8))
    refused(K, -1, "a_scale", quantise(a_scale=P))
    for name in ("a", "codes", "scales"):
        refused(K, -1, f"argument {name} is NULL", quantise(**{name: None}))
        refused(K, -3, f"argument {name}", quantise(**{name: ODD}))

    def dequantise(rows=24, K_=64, dtype=0, codes=P, scales=P, out=P):
        return K._lib.clt_mx4_dequantise(None, 2, rows, K_, dtype, codes, scales, out)
    refused(K, -2, "shape", dequantise(rows=0))
    refused(K, -1, "dtype", dequantise(dtype=5))
    for name in ("codes", "scales", "out"):
        refused(K, -1, f"argument {name} is NULL", dequantise(**{name: None}))
        refused(K, -3, f"argument {name}", dequantise(**{name: ODD}))

    def product(L=2, M=5, N=24, K_=64, ac=P, as_=P, bc=P, bs=P, bias=None, theta=None, dtype=0, out=P):
        return K._lib.clt_mx4_product(None, L, M, N, K_, ac, as_, bc, bs, bias, theta, dtype, out)
    refused(K, -2, "multiple of 8", product(N=20))
    for bad in (dict(M=0), dict(N=0), dict(K_=4), dict(L=0)):
        refused(K, -2, "shape", product(**bad))
    refused(K, -1, "dtype", product(dtype=9))
    for name in ("ac", "as_", "bc", "bs", "out"):
        refused(K, -1, "is NULL", product(**{name: None}))
        refused(K, -3, "aligned", product(**{name: ODD}))
    refused(K, -3, "bias", product(bias=ODD))
    refused(K, -3, "theta", product(theta=ODD))


def test_binding_refuses_what_is_not_on_the_device(K):
    x, w = torch.zeros(2, 3, 64), torch.ones(2, 64)
    for call in (lambda: K.clt_rms_norm(x, w, 1e-5, y=x), lambda: K.clt_rms_norm(None, w, 1e-5), lambda: K.clt_rms_norm(x[0], w, 1e-5),
                 lambda: K.clt_rms_norm(x.double(), w, 1e-5), lambda: K.clt_rms_norm_backward(x, w, x[..., 0], x, x),
                 lambda: K.AdamWTensor(w, w, w, w), lambda: K.AdamWTensor(w, w, w, w, m_scale=w), lambda: K.AdamWTensor(w.int(), w, w, w),
                 lambda: K.AdamW.moments(w, 16), lambda: K.clt_mx4_quantise(x, w, w), lambda: K.clt_mx4_quantise(x[0].to(torch.int8), w, w),
                 lambda: K.clt_mx4_quantise(None, w, w), lambda: K.clt_mx4_dequantise(w, w, x), lambda: K.clt_mx4_product(w, w, w, w, x, 64)):
        with pytest.raises(ValueError):
            call()
    m, v, ms, vs = K.AdamW.moments(torch.zeros(5, 60), 8)
    assert m.shape == v.shape == (5, 60) and m.dtype == torch.uint8 and ms.numel() == vs.numel() == 3
    assert K.AdamW.moments(w)[0].dtype == torch.float32 and K.AdamW.moments(w)[2] is None


# ---- the oracle -------------------------------------------------------------------------------------------------------

def test_oracle_rms_norm_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, w, g, e = rng.normal(size=(2, 3, 16)), 1 + 0.3 * rng.normal(size=(2, 16)), rng.normal(size=(2, 3, 16)), rng.normal(size=(2, 3, 16))

    def f(x, w):      # in 64 bits throughout (the oracle's forward takes 32-bit values)
        r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-3)
        return (x * r * w[:, None, :] * g).sum() + (x * e).sum()
    rstd = 1.0 / np.sqrt((x * x).mean(-1) + 1e-3)
    dx, dw = R.rms_norm_backward(x, w, rstd, g, e)
    for a, da, which in ((x, dx, 0), (w, dw, 1)):
        num = np.zeros_like(a)
        for i in np.ndindex(*a.shape):
            up, down = a.copy(), a.copy()
            up[i] += 1e-6
            down[i] -= 1e-6
            num[i] = (f(up, w) - f(down, w)) / 2e-6 if which == 0 else (f(x, up) - f(x, down)) / 2e-6
        np.testing.assert_allclose(da, num, rtol=1e-7, atol=1e-8)


def test_oracle_formats_against_torch():
    codes = np.arange(128)
    t = torch.arange(128, dtype=torch.uint8)
    assert np.array_equal(R.E4M3.value(codes[:127]), t.view(torch.float8_e4m3fn).double().numpy()[:127])
    assert np.array_equal(R.E5M2.value(codes[:124]), t.view(torch.float8_e5m2).double().numpy()[:124])
    x = np.concatenate([np.float32(1.0) + np.arange(40000, dtype=np.float32) * np.float32(2.0 ** -16), np.float32([1e-30, 3.0e38, -2.5])])
    assert np.array_equal(R.round_bf16(x), torch.from_numpy(x).bfloat16().float().numpy())


@pytest.mark.parametrize("fmt", [R.E4M3, R.E5M2])
def test_oracle_rounding_stays_between_neighbours_and_is_unbiased(fmt):
    rng = np.random.default_rng(5)
    x = np.exp(rng.normal(size=(50, 128)) * 4).astype(np.float32)
    x[:, 0] = 0.0
    s = fmt.block_scale(x)[:, None]
    lo, hi = fmt.encode(x, s, 0.0), fmt.encode(x, s, 1.0 - 2.0 ** -17)
    scale = np.ldexp(1.0, s.astype(int) - 127)
    assert np.all(fmt.value(lo) * scale <= x) and np.all((hi - lo == 1) | (fmt.value(lo) * scale == x) | (hi == lo))
    assert hi.max() <= (0x7E if fmt is R.E4M3 else 0x7B) and np.all(hi[:, 0] == 0)
    n = 4096      # equidistant random numbers: the mean is exact up to half of their distance times the step
    mean = np.mean([fmt.value(fmt.encode(x, s, (i + 0.5) / n)) for i in range(n)], axis=0) * scale
    step = (fmt.value(lo + 1) - fmt.value(lo)) * scale
    # (+ 2^-23 of the smallest normal number of the block, where the 32-bit image of a scaled value ends)
    assert np.all(np.abs(mean - x) <= step / n + np.ldexp(scale, 1 - fmt.bias - 23))


def test_oracle_random_bits_are_uniform_and_differ_between_steps_and_tensors():
    n = 1 << 16
    a = R.random_bits(7, 10, 0, n)
    for b in (R.random_bits(7, 11, 0, n), R.random_bits(7, 10, 1, n), R.random_bits(8, 10, 0, n), R.random_bits(7 + (1 << 32), 10, 0, n),
              R.random_bits(7, 10 + (1 << 32), 0, n), R.random_bits(7, 10, 0, n, first=1 << 32)):
        assert np.mean(a == b) < 1e-3
        c = np.corrcoef((a & np.uint64(0xFFFF)).astype(float), (b & np.uint64(0xFFFF)).astype(float))[0, 1]
        assert abs(c) < 5 / np.sqrt(n)
    for half in (a & np.uint64(0xFFFF), a >> np.uint64(16)):
        # 256 bins of 256 expected: chi-square with 255 degrees of freedom, mean 255, standard deviation 22.6
        chi = ((np.bincount((half >> np.uint64(8)).astype(int), minlength=256) - n / 256) ** 2 / (n / 256)).sum()
        assert 255 - 6 * 22.6 < chi < 255 + 6 * 22.6
        assert abs(np.corrcoef(half[:-1].astype(float), half[1:].astype(float))[0, 1]) < 5 / np.sqrt(n)


def test_second_moment_in_8_bits_follows_the_gradient():
    """2000 steps on gradients of one size: the stored second moments have the right mean and stay near it.  (Rounded to
    nearest they would stop moving at a few per cent of it: 0.1 % a step against grid steps of 14 to 25 %.)"""
    rng = np.random.default_rng(11)
    n, b2 = 512, 0.99      # a memory of 100 steps
    v, vs = np.zeros(n, np.uint8), np.zeros(n // 128, np.uint8)
    m, ms = np.zeros(n, np.uint8), np.zeros(n // 128, np.uint8)
    seen = []
    for t in range(1, 1001):
        o = R.adamw(np.zeros(n), (3e-4 * rng.normal(size=n)).astype(np.float32), m, v, t, 0.0, 0.9, b2, 1e-8, 0.0, ms, vs, 5, 2)
        m, v, ms, vs = o["m"], o["v"], o["m_scale"], o["v_scale"]
        if t > 500:
            seen.append(R.decode_moments(v, vs, R.E5M2, False).astype(np.float64) / 9e-8)
    seen = np.array(seen)
    # rounding noise per step about r * drift with r = 0.19, drift 0.01 * sqrt(2): variance 0.0027 / (2 * 0.01) = 0.13 and 0.01 of the
    # gradients' own; over 512 elements and 500 steps (5 memories): the mean's deviation is sqrt(0.14 / (512 * 2.5)) = 0.0105
    assert abs(seen.mean() - 1.0) < 5 * 0.0105, seen.mean()
    assert seen.std() < 0.6


def test_second_moment_in_8_bits_follows_the_gradient_at_a_memory_of_1000_steps():
    """The same at beta2 = 0.999, where v moves by a thousandth of itself in a step: 6000 steps, the last 3000 looked at."""
    rng = np.random.default_rng(12)
    n, b2 = 512, 0.999
    m, v, ms, vs = np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(n // 128, np.uint8), np.zeros(n // 128, np.uint8)
    total, square = np.zeros(n), 0.0
    for t in range(1, 6001):
        o = R.adamw(np.zeros(n), (3e-4 * rng.normal(size=n)).astype(np.float32), m, v, t, 0.0, 0.9, b2, 1e-8, 0.0, ms, vs, 6, 1)
        m, v, ms, vs = o["m"], o["v"], o["m_scale"], o["v_scale"]
        if t > 3000:
            x = R.decode_moments(v, vs, R.E5M2, False).astype(np.float64) / 9e-8 / (1.0 - b2 ** t)
            total += x
            square += (x * x).mean()
    mean = total.mean() / 3000
    # rounding to a neighbour: variance (grid step) * |drift| = 0.19 * 0.001 * E|g^2 - 1| (0.97) = 1.8e-4 a step, over 2 * 0.001: 0.092, and 0.001 of
    # the gradients' own; over 512 elements and 3 memories, with a correlation over two of them: sqrt(0.093 * 2 / 3 / 512) = 0.011
    assert abs(mean - 1.0) < 5 * 0.011, mean
    assert np.sqrt(square / 3000 - mean ** 2) < 0.45      # (0.31 expected)


def test_oracle_mx4_packing_and_rounding():
    rng = np.random.default_rng(9)
    a = (rng.normal(size=(2, 70, 200)) * np.exp(2 * rng.normal(size=(2, 70, 1)))).astype(np.float32)
    a[0, 3, :32] = 0.0
    codes, s = R.mx4_round(a)
    assert codes.shape == (2, 70, 256) and s.shape == (2, 70, 8)
    pc, ps = R.mx4_pack(codes, s)
    c2, s2 = R.mx4_unpack(pc, ps, 70)
    assert np.array_equal(codes, c2) and np.array_equal(s, s2)
    v = R.mx4_values(codes, s)[..., :200]
    top = np.abs(np.pad(a, ((0, 0), (0, 0), (0, 56))).reshape(2, 70, 8, 32)).max(-1)
    unit = np.ldexp(1.0, s.astype(int) - 127).repeat(32, -1)[..., :200]
    x = np.abs(a) / unit
    half = np.where(x < 2, 0.25, np.where(x < 4, 0.5, 1.0)) * unit
    assert np.all(np.abs(v - a) <= half)                      # never off by more than half a step
    assert np.all(top[s > 0] / np.ldexp(1.0, s[s > 0].astype(int) - 127) >= 3.5)      # and no smaller power would do
    # ties go to the even code, saturation and signs
    ties = np.zeros((1, 1, 32), np.float32)
    ties[0, 0, :12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5, 6.9, 6.99]
    assert R.mx4_values(*R.mx4_round(ties))[0, 0, :12].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -4, 6, 6]
    bad = np.zeros((1, 2, 32), np.float32)
    bad[0, 0, 5], bad[0, 1, 6] = np.nan, -np.inf
    assert R.mx4_round(bad)[1][0, :, 0].tolist() == [255, 255]


# ---- the optimiser inside the training step: what it may be given -------------------------------------------------------

class _Step:
    """A CLTStep without a device: tensors on the host, and its GPU calls written down instead of made."""

    def __new__(cls, K, **config):
        step = object.__new__(K.CLTStep)
        L, d, F, B = 2, 64, 136, 8
        step.cfg = K.make_config(L, d, F, B, K.DTYPE_BF16, **config)
        step.adam = (0.9, 0.999, 1e-8)
        f32, T = torch.float32, torch.bfloat16
        step.grads = {"b_enc": torch.zeros(L, F), "theta": torch.zeros(L, F), "b_dec": torch.zeros(L, d), "W_enc": torch.zeros(L, d, F, dtype=T),
                      "W_dec": torch.zeros(3, F, d, dtype=T)}
        step.calls = []
        for name in ("forward", "loss", "backward", "backward_adam_step", "adam_step"):
            setattr(step, name, lambda *a, name=name, **k: step.calls.append(name))
        return step


def test_adamw_of_a_step_with_master_weights_needs_them(K, monkeypatch):
    made = []
    monkeypatch.setattr(K, "AdamWTensor", lambda *a: made.append(a))
    monkeypatch.setattr(K, "AdamW", type("List", (), {"__init__": lambda self, *a: None, "moments": K.AdamW.moments}))
    step = _Step(K, master_weights=True)
    params = {k: g.clone() for k, g in step.grads.items()}
    master = {k: params[k].float() for k in ("W_enc", "W_dec")}
    for bad in (None, {}, {"W_enc": master["W_enc"]}, {"W_dec": master["W_dec"]}, dict(master, W_enc=None)):
        with pytest.raises(ValueError, match="master"):
            step.adamw(params, master=bad)
    assert not made
    step.adamw(params, master=master)
    assert [a[6] is not None for a in made] == [False, False, False, True, True]
    made.clear()      # without the flag they may be left out
    _Step(K).adamw(params)
    assert [a[6] for a in made] == [None] * 5


def test_train_step_takes_an_optimiser_of_its_own_parameters_only(K):
    step = _Step(K)
    params = {k: g.clone() for k, g in step.grads.items()}

    def optimiser(p, g):
        """An AdamW over p and g; steps are written down."""
        opt = object.__new__(K.AdamW)
        opt.tensors = [types.SimpleNamespace(c=K.clt_adamw_tensor(p=p[k].data_ptr(), g=g[k].data_ptr())) for k in p]
        opt.step = lambda t, lr: step.calls.append("adamw")
        return opt

    def train(opt):
        step.calls.clear()
        step.train_step(None, None, params, None, None, 1, 1e-3, 1.0, optimiser=opt)
    other = {k: p.clone() for k, p in params.items()}
    for bad in (optimiser(other, step.grads),                                       # the forward pass would read what no step writes
                optimiser(dict(params, W_dec=other["W_dec"]), step.grads),
                optimiser(params, {k: g.clone() for k, g in step.grads.items()}),   # gradients of another step
                optimiser({}, {})):
        with pytest.raises(ValueError, match="optimiser"):
            train(bad)
        assert not step.calls
    train(optimiser(params, step.grads))
    assert step.calls == ["forward", "loss", "backward", "adamw"]
    # a part of the parameters, or others beside them, are the caller's choice
    train(optimiser({"W_enc": params["W_enc"]}, step.grads))
    train(optimiser(dict(params, more=other["W_enc"]), dict(step.grads, more=other["W_dec"])))
    old = optimiser(params, step.grads)
    params["W_enc"] = params["W_enc"].clone()      # other memory than the list was made for
    with pytest.raises(ValueError, match="optimiser"):
        train(old)
    step.calls.clear()
    step.train_step(None, None, params, None, None, 1, 1e-3, 1.0, fused=False)
    assert step.calls == ["forward", "loss", "backward", "adam_step"]
