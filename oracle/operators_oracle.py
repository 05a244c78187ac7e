"""CPU oracle of the operators around the training step (test infrastructure only): RMS norm with its gradients, AdamW with
moments in 32 or 8 bits, matrices in 4-bit microscaled floating point.  Plain numpy in 64 bits; where a result is decided by
a 32-bit rounding (the moments, whose codes are compared bit for bit) the 32-bit operations are written out one by one."""
import numpy as np

BLOCK8 = 128      # elements that share a scale, 8-bit moments


def round_bf16(x):
    """Nearest bf16 (ties to even) of finite float32 values, as float32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)).view(np.float32)


# ---- RMS norm --------------------------------------------------------------------------------------------------------

def rms_norm(x, weight, eps, residual=None, bf16=False):
    """x, residual [L,B,d] float32 arrays (storage values), weight [L,d]: (h, rstd, y) with y unrounded."""
    h = np.asarray(x, dtype=np.float32)
    if residual is not None:
        h = h + np.asarray(residual, dtype=np.float32)
        if bf16:
            h = round_bf16(h)
    h64 = h.astype(np.float64)
    rstd = 1.0 / np.sqrt((h64 * h64).mean(-1) + eps)
    return h, rstd, h64 * rstd[..., None] * np.asarray(weight, dtype=np.float64)[:, None, :]


def rms_norm_backward(h, weight, rstd, dy, dh=None):
    """(dx, dweight) for rstd as the forward pass gave it."""
    h, w, r, g = (np.asarray(a, dtype=np.float64) for a in (h, weight, rstd, dy))
    r, w = r[..., None], w[:, None, :]
    dx = r * w * g - h * r ** 3 * (w * g * h).mean(-1, keepdims=True)
    return dx if dh is None else dx + np.asarray(dh, dtype=np.float64), (g * h * r).sum(1)


# ---- AdamW -----------------------------------------------------------------------------------------------------------

def mix32(x):
    x = np.asarray(x, dtype=np.uint64) & 0xFFFFFFFF
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x9E3779B1)) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x85A308D3)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(seed, t, index, n, first=0):
    """32 random bits for each of n elements (from element `first`) of the list's tensor `index` at step t."""
    key_t = int(mix32(t >> 32)) ^ (t & 0xFFFFFFFF)
    key = int(mix32((seed & 0xFFFFFFFF) ^ int(mix32((seed >> 32) ^ int(mix32(key_t ^ int(mix32(index + 0x243F6A88))))))))
    i = np.arange(first, first + n, dtype=np.uint64)
    return mix32((i & np.uint64(0xFFFFFFFF)) ^ ((key + (i >> np.uint64(32)) * np.uint64(0x85A308D3)) & np.uint64(0xFFFFFFFF)))


class Float8:
    """An 8-bit float: mantissa bits, exponent bias, exponent of the largest finite value (1.75 times that power)."""

    def __init__(self, mantissa, bias, top):
        self.mantissa, self.bias, self.top = mantissa, bias, top

    def value(self, code):
        """Of codes without a sign."""
        code = np.asarray(code, dtype=np.int64)
        e, f = code >> self.mantissa, code & ((1 << self.mantissa) - 1)
        frac = f / float(1 << self.mantissa)
        return np.where(e == 0, np.ldexp(frac, 1 - self.bias), np.ldexp(1.0 + frac, e - self.bias))

    def block_scale(self, x):
        """Scale byte of one block of non-negative float32 values (any shape, last axis the block)."""
        top = np.asarray(x, dtype=np.float64).max(-1)
        broken = ~np.isfinite(np.asarray(x, dtype=np.float64)).all(-1)
        top = np.where(broken, 1.0, top)
        f, e = np.frexp(top)                            # top = f 2^e, 1/2 <= f < 1
        e = np.where(f > 0.875, e + 1, e) - 1           # the power below it, or the next one where it exceeds 1.75 of that
        s = np.maximum(np.where(top > 0, e + 127, 0) - self.top, 0)
        return np.where(broken | (e + 127 >= 255), 255, s).astype(np.uint8)

    def encode(self, x, s, uniform):
        """Codes of float32 x >= 0 in blocks with scale s: the neighbour below, or with probability `distance` the one above."""
        y = np.ldexp(np.asarray(x, dtype=np.float64), 127 - s.astype(np.int64))
        _, e = np.frexp(y)
        e = np.where(y > 0, np.maximum(e - 1, 1 - self.bias), 1 - self.bias)
        # (2^-23 of the smallest normal number is where the scaled fp32 image ends)
        y = np.where(y < np.ldexp(1.0, 1 - self.bias), np.round(np.ldexp(y, self.bias - 1 + 23)) * np.ldexp(1.0, 1 - self.bias - 23), y)
        steps = np.floor(np.ldexp(y, self.mantissa - e) + uniform).astype(np.int64)
        return np.where(s == 255, 0, steps + ((e - (1 - self.bias)) << self.mantissa)).astype(np.int64)


E4M3, E5M2 = Float8(3, 7, 8), Float8(2, 15, 15)


def _blocks(a, fill=0):
    a = np.asarray(a).reshape(-1)
    return np.pad(a, (0, -a.size % BLOCK8), constant_values=fill).reshape(-1, BLOCK8)


def decode_moments(code, s, fmt, signed):
    """float32 values of 8-bit moments."""
    code, n = np.asarray(code, dtype=np.uint8), np.asarray(code).size
    sign = np.where(_blocks(code) & 0x80, -1.0, 1.0) if signed else 1.0
    x = sign * np.ldexp(fmt.value(_blocks(code) & (0x7F if signed else 0xFF)), s.astype(np.int64)[:, None] - 127)
    x = np.where(s[:, None] == 255, np.nan, x)
    return x.astype(np.float32).reshape(-1)[:n]


def adamw(p, g, m, v, t, lr, b1, b2, eps, decay, m_scale=None, v_scale=None, seed=0, index=0):
    """One step on flat float32 arrays (p: the master copy or the values of p); returns a dict with p in 64 bits, unrounded, the
    32-bit moments before 8-bit rounding (m32, v32), and m, v (and scales) as stored."""
    f = np.float32
    g = np.asarray(g, dtype=f)
    eight = m_scale is not None
    if eight:
        m, v = decode_moments(m, m_scale, E4M3, True), decode_moments(v, v_scale, E5M2, False)
    with np.errstate(over="ignore", invalid="ignore", under="ignore"):
        m = f(b1) * np.asarray(m, dtype=f) + f(1.0 - b1) * g
        v = f(b2) * np.asarray(v, dtype=f) + (f(1.0 - b2) * g) * g
        den = np.sqrt(v.astype(np.float64) / (1.0 - b2 ** t)) + eps
        p = np.asarray(p, dtype=np.float64) * (1.0 - lr * decay) - lr / (1.0 - b1 ** t) * m.astype(np.float64) / den
    out = {"p": p, "m32": m, "v32": v, "m": m, "v": v}
    if eight:
        n = g.size
        r = random_bits(seed, t, index, n)
        um, uv = ((r & np.uint64(0xFFFF)).astype(np.float64) + 0.5) / 65536, ((r >> np.uint64(16)).astype(np.float64) + 0.5) / 65536
        mb, vb = _blocks(np.abs(m)), _blocks(v)
        out["m_scale"], out["v_scale"] = E4M3.block_scale(mb), E5M2.block_scale(vb)
        mb, vb = np.nan_to_num(mb, posinf=0.0), np.nan_to_num(vb, posinf=0.0)
        mc = E4M3.encode(mb, out["m_scale"][:, None], _blocks(um)) | np.where(_blocks(m) < 0, 0x80, 0)
        vc = E5M2.encode(vb, out["v_scale"][:, None], _blocks(uv))
        vc = np.where((vb > 0) & (vc == 0) & (out["v_scale"][:, None] != 255), 1, vc)
        out["m"], out["v"] = (c.reshape(-1)[:n].astype(np.uint8) for c in (mc, vc))
    return out


# ---- 4-bit microscaled floating point ------------------------------------------------------------------------------------

FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_round(a):
    """a [..., K] float32 values -> (codes [..., KP], scale bytes [..., KP / 32]), K padded to KP, a multiple of 128."""
    a = np.asarray(a, dtype=np.float64)
    K = a.shape[-1]
    a = np.pad(a, [(0, 0)] * (a.ndim - 1) + [(0, -K % 128)]).reshape(*a.shape[:-1], -1, 32)
    broken = ~np.isfinite(a).all(-1)
    a = np.where(broken[..., None], 0.0, a)
    top = np.abs(a).max(-1)
    f, e = np.frexp(top)
    # (numbers below 2^-126 lie on the grid of the smallest exponent)
    s = np.where(top > 0, np.where(f >= 0.875, e, e - 1) + 127 - 2, 0)
    s = np.where(broken, 255, np.maximum(s, 0)).astype(np.uint8)
    x = np.abs(np.ldexp(a, 127 - np.where(broken, 127, s).astype(np.int64)[..., None]))
    # nearest of the eight magnitudes; of two equally near ones the even code
    d = np.abs(x[..., None] - FP4)
    near = d == d.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = code | np.where(np.signbit(a), 8, 0)
    return code.reshape(*code.shape[:-2], -1).astype(np.uint8), s


def mx4_values(codes, s):
    v = FP4[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    v = v.reshape(*s.shape, 32) * np.where(s == 255, np.nan, np.ldexp(1.0, s.astype(np.int64) - 127))[..., None]
    return v.reshape(codes.shape)


def mx4_pack(codes, s):
    """[L, rows, KP] codes, [L, rows, KP/32] scales -> the packed arrays of include/clt.h, element by element."""
    L, R, KP = codes.shape
    RP, KS = (R + 63) // 64, KP // 128
    pc, ps = np.zeros((L, 4 * RP, KS, 1024), np.uint8), np.zeros((L, RP, KS, 256), np.uint8)
    r = np.arange(R)
    for k in range(KP):
        at = ((k % 128) // 32 * 16 + r % 16) * 16 + (k % 32) // 2
        pc[:, r // 16, k // 128, at] |= codes[:, :, k] << (4 * (k % 2))
    for b in range(KP // 32):
        ps[:, r // 64, b // 4, (b % 4 * 16 + r % 16) * 4 + r % 64 // 16] = s[:, :, b]
    return pc, ps


def mx4_unpack(pc, ps, R):
    """The packed arrays -> (codes [L, R, KP], scales [L, R, KP/32])."""
    L, _, KS, _ = pc.shape
    r, k = np.arange(R)[:, None], np.arange(KS * 128)[None, :]
    byte = pc[:, r // 16, k // 128, ((k % 128) // 32 * 16 + r % 16) * 16 + (k % 32) // 2]
    b = np.arange(KS * 4)[None, :]
    return (byte >> (4 * (k % 2)).astype(np.uint8)) & 15, ps[:, r // 64, b // 4, (b % 4 * 16 + r % 16) * 4 + r % 64 // 16]
