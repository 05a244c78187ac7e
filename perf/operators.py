"""What is timed of the operators around the training step: the RMS norm that makes its 8-bit inputs, the AdamW step with states
in 8 or 32 bits, and the encoder in 4-bit microscaled floating point.

A case holds
  kind   norm           h = x + residual, RMS norm of h, as the storage type or as int8 codes with one scale per row
         norm_backward  gradients of that norm with respect to h and to the weights
         adamw          one AdamW step on the five tensors of a transcoder
         mx4_quantise   rows (or a weight matrix, transposed) to 4 bits and back
         mx4_encode     activations to 4 bits and their product with 4-bit encoder weights, bias and threshold
  L B d F     layers, tokens of the batch, model width, features per layer
  dtype       bf16 | f32 storage of activations and matrices
  residual    norm: a residual is added;  norm_backward: a gradient reaches h past the norm
  int8        norm: int8 codes come out;  mx4_quantise: int8 codes with row scales come in
  states      adamw: bits of the matrices' moments (8 | 32);  master: fp32 master copies of the matrices;  decay: weight decay
  transposed  mx4_quantise: an encoder weight [d, F] whose blocks run along d
  theta       mx4_encode: threshold of the activation (0: plain pre-activations)

Plain forms and kernels take the same state.  Packed 4-bit operands are laid out as include/clt.h documents them.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS, B1, B2, ADAM_EPS, LR, FIRST_STEP, SEED = 1e-5, 0.9, 0.999, 1e-8, 2e-4, 1001, 20240601
MATRICES = ("W_enc", "W_dec")
GRADIENT = 1e-3      # size of gradients and of their running moments


def _case(name, kind, L, B, d, F=0, dtype="bf16", residual=False, int8=False, states=0, master=False, decay=0.0, transposed=False,
          theta=0.0):
    return {"name": name, "kind": kind, "L": L, "B": B, "d": d, "F": F, "dtype": dtype, "residual": residual, "int8": int8,
            "states": states, "master": master, "decay": decay, "transposed": transposed, "theta": theta}


def listed():
    return [
        # one token on its way through a layer: latency alone
        _case("norm_token", "norm", 1, 1, 2048, residual=True),
        # MLP inputs of an odd batch in full precision, straight into the int8 cache format
        _case("norm_gpt2_f32_int8", "norm", 12, 1037, 768, dtype="f32", int8=True),
        # the residual streams of a training batch into the int8 inputs of the step
        _case("norm_llama1b_int8", "norm", 16, 4096, 2048, residual=True, int8=True),
        # gradients of a short odd batch in one layer, a width that fits no power of two
        _case("norm_backward_ragged", "norm_backward", 1, 300, 2056),
        # gradients of a training batch, with the residual's own gradient
        _case("norm_backward_llama1b", "norm_backward", 16, 4096, 2048, residual=True),
        # the smallest transcoder (unit tests, notebooks): five tensors, launches
        _case("adamw_tiny_8bit", "adamw", 4, 0, 64, 256, dtype="f32", states=8),
        # the GPT-2 transcoder with moments in 32 bits
        _case("adamw_gpt2_32bit", "adamw", 12, 0, 768, 6144, states=32, decay=0.01),
        # half of the Llama transcoder's layers with moments in 8 bits
        _case("adamw_llama1b_half_8bit", "adamw", 8, 0, 2048, 8192, states=8, decay=0.01),
        # a batch of the int8 cache into 4 bits, sizes that fit no tile
        _case("mx4_cache_ragged", "mx4_quantise", 6, 1037, 2056, int8=True),
        # encoder weights of the GPT-2 transcoder into 4 bits, blocks along the contraction
        _case("mx4_weights_gpt2", "mx4_quantise", 12, 0, 768, 6144, transposed=True),
        # features of one token of a prompt, all layers: bound by the weights
        _case("mx4_encode_token", "mx4_encode", 16, 1, 2048, 8192, theta=0.03),
        # encoder-only pass over a batch (feature statistics over many tokens)
        _case("mx4_encode_llama1b", "mx4_encode", 16, 4096, 2048, 8192, theta=0.03),
    ]


def _log_between(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _multiple_of_8(x, rng):
    n = max(8, int(round(x / 8)) * 8)
    if n >= 256 and rng.random() < 0.5:      # half of the wide ones are the round sizes that models have
        n = n // 256 * 256
    return n


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "adamw", "mx4_quantise", "mx4_encode", "mx4_encode"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    while True:
        L = int(round(_log_between(rng, 1, 16)))
        d = _multiple_of_8(_log_between(rng, 64, 4096), rng)
        F = _multiple_of_8(d * _log_between(rng, 2, 16), rng) if kind in ("adamw", "mx4_quantise", "mx4_encode") else 0
        B = int(round(_log_between(rng, 1, 16384)))
        if rng.random() < 0.4 and B >= 64:
            B = B // 64 * 64
        transposed = kind == "mx4_quantise" and rng.random() < 0.5
        if kind == "adamw":
            B = 0
            if F <= 16384 and (L * (L + 1) // 2 + L) * F * d <= 5e8:
                break
        elif kind == "mx4_encode":
            if F <= 32768 and L * B * F * 1.0 <= 4.5e8 and L * d * F <= 2.7e8 and 2.0 * L * B * F * d <= 1.6e12:
                break
        elif kind == "mx4_quantise":
            B, F = (0, F) if transposed else (B, 0)
            if F <= 32768 and L * d * (F or B) * 1.0 <= 1.3e8:
                break
        elif L * B * d * 1.0 <= (6.5e7 if dtype == "f32" else 1.3e8):
            break
    c = _case("", kind, L, B, d, F, dtype)
    c["residual"] = kind in ("norm", "norm_backward") and rng.random() < 0.6
    c["int8"] = kind == "norm" and rng.random() < 0.6 or kind == "mx4_quantise" and not transposed and rng.random() < 0.5
    if kind == "mx4_quantise" and c["int8"]:
        c["dtype"] = "bf16"
    c["transposed"] = transposed
    if kind == "adamw":
        c["states"] = rng.choice([8, 8, 32])
        c["master"] = dtype == "bf16" and rng.random() < 0.3
        c["decay"] = rng.choice([0.0, 0.01, 0.1])
    if kind == "mx4_encode":
        c["theta"] = rng.choice([0.0, 0.03])
    del c["name"]
    return c


# ---- what a program has in hand before the call --------------------------------------------------------------------

def _shapes(case):
    L, d, F = case["L"], case["d"], case["F"]
    return {"W_enc": (L, d, F), "b_enc": (L, F), "theta": (L, F), "W_dec": (L * (L + 1) // 2, F, d), "b_dec": (L, d)}


def _panels(rows, K):
    """Sizes of a packed 4-bit operand: panels of 64 rows, steps of 128 elements of the contraction."""
    return (rows + 63) // 64, (K + 127) // 128


def _pack(w):
    """[L, rows, K] float -> packed codes and scales (include/clt.h), made here because a program that serves an encoder has them
    from its checkpoint."""
    L, R, K = w.shape
    rp, kp = _panels(R, K)
    w = torch.nn.functional.pad(w, (0, kp * 128 - K, 0, rp * 64 - R)).view(L, rp * 64, kp, 4, 32)
    amax = w.abs().amax(-1)
    e = torch.floor(torch.log2((amax * (8.0 / 7.0)).clamp_min(1e-30))).clamp_min(-100.0) - 2.0
    a = w.abs() * torch.exp2(-e)[..., None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    code += 8 * (w < 0).to(torch.uint8)
    code = (code[..., 0::2] + 16 * code[..., 1::2]).view(L, rp * 4, 16, kp, 4, 16)      # layer, 16 rows, row, step, block, byte
    scale = (e + 127.0).to(torch.uint8).view(L, rp, 4, 16, kp, 4)                       # layer, 64 rows, 16 rows, row, step, block
    return (code.permute(0, 1, 3, 4, 2, 5).reshape(L, rp * 4, kp, 1024).contiguous(),
            scale.permute(0, 1, 4, 5, 3, 2).reshape(L, rp, kp, 256).contiguous())


def _moments_in_8_bits(m, v):
    """Codes and block scales of running moments (nearest is near enough for a state to begin with)."""
    n = m.numel()
    blocks = (n + 127) // 128

    def one(x, top, T):
        x = torch.nn.functional.pad(x.reshape(-1), (0, blocks * 128 - n)).view(blocks, 128)
        amax = x.abs().amax(1).clamp_min(1e-30)
        s = torch.floor(torch.log2(amax * (8.0 / 7.0))) - top
        code = (x * torch.exp2(-s)[:, None]).to(T).view(torch.uint8).reshape(-1)[:n].clone()
        return code, (s + 127.0).to(torch.uint8)
    m8, ms = one(m, 8, torch.float8_e4m3fn)
    v8, vs = one(v, 15, torch.float8_e5m2)
    return m8, v8, ms, vs


def prepare(case, seed):
    L, B, d, F, kind = case["L"], case["B"], case["d"], case["F"], case["kind"]
    T = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    def empty(*shape, dtype=T):
        return torch.empty(shape, dtype=dtype, device=DEVICE)

    s = {"case": case}
    if kind in ("norm", "norm_backward"):
        # residual streams: norms that grow with depth, spread over the tokens, a few outlier dimensions; norm weights near one
        x = normal(L, B, d) * (1.0 + 0.25 * torch.arange(L, device=DEVICE))[:, None, None] * torch.exp(0.5 * normal(B))[None, :, None]
        x[:, :, torch.randperm(d, generator=g, device=DEVICE)[:4]] *= 20.0
        s["x"] = x.to(T)
        del x
        s["weight"] = 1.0 + 0.2 * normal(L, d)
        if kind == "norm":
            s["residual"] = (0.5 * normal(L, B, d)).to(T) if case["residual"] else None
            s["h"] = empty(L, B, d) if case["residual"] else None
            s["rstd"], s["scale"] = empty(L, B, dtype=torch.float32), empty(L, B, dtype=torch.float32)
            s["q"] = empty(L, B, d, dtype=torch.int8) if case["int8"] else None
            s["y"] = empty(L, B, d, dtype=torch.bfloat16 if case["int8"] else T)
        else:
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(-1) + EPS)
            s["dy"], s["dx"] = (GRADIENT * normal(L, B, d)).to(T), empty(L, B, d)
            s["dh"] = (GRADIENT * normal(L, B, d)).to(T) if case["residual"] else None
            s["dweight"] = empty(L, d, dtype=torch.float32)
        return s
    if kind == "adamw":
        s["t"], s["tensors"] = FIRST_STEP, {}
        for name, shape in _shapes(case).items():
            matrix = name in MATRICES
            Tp = T if matrix else torch.float32
            w = (torch.rand(shape, generator=g, device=DEVICE) * 2 - 1) / math.sqrt(d)
            if matrix:      # gradients of features that are active to a varying degree
                size = torch.exp(0.7 * normal(*shape[:2]))[..., None]
            else:
                size = 1.0
            q = {"p": w.to(Tp), "g": (GRADIENT * size * normal(*shape)).to(Tp), "master": w if matrix and case["master"] else None}
            del w
            q["m"] = (0.3 * GRADIENT) * size * normal(*shape)
            q["v"] = (torch.rand(shape, generator=g, device=DEVICE) + 0.5) * ((GRADIENT * size) * (GRADIENT * size))
            if matrix and case["states"] == 8:
                q["m"], q["v"], q["m_scale"], q["v_scale"] = _moments_in_8_bits(q["m"], q["v"])
                q["m"], q["v"] = q["m"].view(shape), q["v"].view(shape)
            else:
                q["m_scale"] = q["v_scale"] = None
            q["decay"] = case["decay"] if matrix else 0.0
            s["tensors"][name] = q
        return s
    if kind == "mx4_quantise":
        if case["transposed"]:
            s["a"], s["a_scale"] = ((torch.rand((L, d, F), generator=g, device=DEVICE) * 2 - 1) / math.sqrt(d)).to(T), None
            rows = F
        else:
            x = normal(L, B, d) * torch.exp(0.5 * normal(B))[None, :, None]
            rows = B
            if case["int8"]:
                s["a_scale"] = x.abs().amax(2) / 127.0
                s["a"] = torch.round(x / s["a_scale"][:, :, None]).to(torch.int8)
            else:
                s["a"], s["a_scale"] = x.to(T), None
        rp, kp = _panels(rows, d)
        s["codes"], s["scales"] = empty(L, rp * 4, kp, 1024, dtype=torch.uint8), empty(L, rp, kp, 256, dtype=torch.uint8)
        s["out"] = empty(L, rows, d)
        return s
    x = normal(L, B, d)
    s["x"] = x.to(T)
    s["w_codes"], s["w_scales"] = _pack((torch.rand((L, F, d), generator=g, device=DEVICE) * 2 - 1) / math.sqrt(d))
    s["bias"] = 0.01 * normal(L, F)
    s["theta"] = torch.full((L, F), case["theta"], device=DEVICE) if case["theta"] else None
    rp, kp = _panels(B, d)
    s["x_codes"], s["x_scales"] = empty(L, rp * 4, kp, 1024, dtype=torch.uint8), empty(L, rp, kp, 256, dtype=torch.uint8)
    s["out"] = empty(L, B, F)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _norm(s):
    x, case = s["x"], s["case"]
    T = x.dtype
    h = (x.float() + s["residual"].float()).to(T) if case["residual"] else x
    t = h.float()
    rstd = torch.rsqrt(t.square().mean(-1) + EPS)
    t = t * s["weight"][:, None, :]
    out = {"rstd": rstd}
    if case["residual"]:
        out["h"] = h
    if not case["int8"]:
        out["y"] = (t * rstd[..., None]).to(T)
        return out
    amax = t.abs().amax(-1)
    k = torch.where(amax > 0, 127.0 / amax, torch.zeros_like(amax))
    scale = torch.where(amax > 0, amax * rstd / 127.0, torch.ones_like(amax))
    out["scale"] = scale
    out["y"] = (torch.round(t * k[..., None]) * scale[..., None]).bfloat16()
    return out


def _norm_backward(s):
    h, dy, rstd, w = s["x"].float(), s["dy"].float(), s["rstd"][..., None], s["weight"][:, None, :]
    wdy = w * dy
    c = (wdy * h).mean(-1, keepdim=True)
    dx = rstd * wdy - h * (rstd * rstd * rstd * c)
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * h * rstd).sum(1)}


def _mix(x):
    """A 32-bit mixing function in 64-bit integers: products keep their low 32 bits, whatever wraps above them."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B1) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x85A308D3) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(t, index):
    return _mix((SEED & 0xFFFFFFFF) ^ _mix((SEED >> 32) ^ _mix(t ^ _mix(index + 0x243F6A88))))


def _decode8(code, scale, T):
    """Values of 8-bit moments: elements of type T times the power of two of their block."""
    n = code.numel()
    x = torch.nn.functional.pad(code.reshape(-1), (0, -n % 128)).view(T).float().view(-1, 128)
    return (x * torch.exp2(scale.float() - 127.0)[:, None]).view(-1)[:n]


def _encode8(x, random, mantissa, top):
    """Non-negative 32-bit values to 8-bit floats with one power of two per 128: the image of the float, shifted and cut, is the code;
    random bits below the cut make the rounding unbiased."""
    n = x.numel()
    x = torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)
    e = (x.amax(1).view(torch.int32) + 0x1FFFFF) >> 23
    s = (e - top).clamp_min(0)
    bias = 15 if mantissa == 2 else 7
    y = (x.double() * torch.exp2((bias - s).double())[:, None]).float().view(torch.int32).view(-1)[:n]
    cut = 23 - mantissa
    low = (random << (cut - 16)) | (1 << (cut - 17))
    return (y + low) >> cut, s


def _adamw_one(q, index, t):
    shape = q["p"].shape
    g = q["g"].float().reshape(-1)
    eight = q["m_scale"] is not None
    m = _decode8(q["m"], q["m_scale"], torch.float8_e4m3fn) if eight else q["m"].reshape(-1)
    v = _decode8(q["v"], q["v_scale"], torch.float8_e5m2) if eight else q["v"].reshape(-1)
    m = B1 * m + (1.0 - B1) * g
    v = B2 * v + ((1.0 - B2) * g) * g
    p = (q["master"] if q["master"] is not None else q["p"]).float().reshape(-1)
    p = p * (1.0 - LR * q["decay"]) - (LR / (1.0 - B1 ** t)) * m / ((v / (1.0 - B2 ** t)).sqrt() + ADAM_EPS)
    q["p"].copy_(p.view(shape))
    if q["master"] is not None:
        q["master"].copy_(p.view(shape))
    if not eight:
        q["m"].copy_(m.view(shape))
        q["v"].copy_(v.view(shape))
        return
    del p, g
    h = _mix(torch.arange(m.numel(), device=DEVICE) ^ _key(t, index))
    code, s = _encode8(m.abs(), (h & 0xFFFF).to(torch.int32), 3, 8)
    q["m"].copy_((code | (m < 0).to(torch.int32) << 7).view(shape))
    q["m_scale"].copy_(s)
    code, s = _encode8(v, (h >> 16).to(torch.int32), 2, 15)
    q["v"].copy_(torch.where(v > 0, code.clamp_min(1), code).view(shape))
    q["v_scale"].copy_(s)


def _adamw_outputs(s):
    """Tensors of the step; 8-bit moments as the floats that their elements are, beside the scales of their blocks."""
    out = {}
    for name, q in s["tensors"].items():
        eight = q["m_scale"] is not None
        out[name] = {"p": q["p"], "master": q["master"], "m": q["m"].view(torch.float8_e4m3fn) if eight else q["m"],
                     "v": q["v"].view(torch.float8_e5m2) if eight else q["v"],
                     "m_scale": q["m_scale"].view(torch.float8_e8m0fnu) if eight else None,
                     "v_scale": q["v_scale"].view(torch.float8_e8m0fnu) if eight else None}
    return out


def _round4(x):
    """[..., K] float -> the values that 4-bit elements with a power of two per 32 stand for."""
    K = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -K % 32)).unflatten(-1, (-1, 32))
    e = ((x.abs().amax(-1).view(torch.int32) + 0x200000) >> 23) - 2
    step = torch.exp2((e.clamp_min(0) - 127).double()).float()[..., None]
    a = x.abs() / step
    half = ((a > 0.25).float() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + 2 * (a > 2.5).float() + 2 * (a >= 3.5).float() + 4 * (a > 5.0).float())
    return (torch.copysign(0.5 * half * step, x)).flatten(-2)[..., :K]


def _unpack(codes, scales, rows, K):
    """Packed codes and scales -> [L, rows, K] float."""
    L, rp, kp = scales.shape[:3]
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=DEVICE)
    c = codes.view(L, rp * 4, kp, 4, 16, 16).permute(0, 1, 4, 2, 3, 5)                      # layer, 16 rows, row, step, block, byte
    c = torch.stack((c & 15, c >> 4), -1).int().reshape(L, rp * 64, kp * 4, 32)
    e = scales.view(L, rp, kp, 4, 16, 4).permute(0, 1, 5, 4, 2, 3).reshape(L, rp * 64, kp * 4)
    return (value[c] * torch.exp2(e.float() - 127.0)[..., None]).view(L, rp * 64, kp * 128)[:, :rows, :K]


def _mx4_quantise(s):
    a = s["a"].float()
    if s["a_scale"] is not None:
        a = a * s["a_scale"][..., None]
    if s["case"]["transposed"]:
        a = a.transpose(1, 2).contiguous()
    return {"values": _round4(a).to(s["out"].dtype)}


def _mx4_encode(s):
    case = s["case"]
    w = _unpack(s["w_codes"], s["w_scales"], case["F"], case["d"]).transpose(1, 2).contiguous()
    pre = torch.bmm(_round4(s["x"].float()), w) + s["bias"][:, None, :]
    if s["theta"] is not None:
        pre = pre * (pre > s["theta"][:, None, :])
    return {"z": pre.to(s["out"].dtype)}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, case, kind)
    if kind == "norm":
        return _norm(s)
    if kind == "norm_backward":
        return _norm_backward(s)
    if kind == "mx4_quantise":
        return _mx4_quantise(s)
    if kind == "mx4_encode":
        return _mx4_encode(s)
    [_adamw_one(q, k, s["t"]) for k, q in enumerate(s["tensors"].values())]
    s["t"] += 1
    return _adamw_outputs(s)


def _run_own(s, case, kind):
    from paper_2603_21014_amd import binding as K
    if kind == "norm":
        int8 = case["int8"]
        K.clt_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], h=s["h"], y=None if int8 else s["y"], q=s["q"],
                       q_scale=s["scale"] if int8 else None, rstd=s["rstd"])
        out = {"rstd": s["rstd"]}
        if case["residual"]:
            out["h"] = s["h"]
        if int8:      # the values that the codes stand for
            out["scale"] = s["scale"]
            out["y"] = torch.mul(s["q"], s["scale"][..., None], out=s["y"])
        else:
            out["y"] = s["y"]
        return out
    if kind == "norm_backward":
        if "workspace" not in s:      # kept by a program between its steps
            n = K.clt_rms_norm_backward_workspace_bytes(case["L"], case["B"], case["d"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEVICE)
        K.clt_rms_norm_backward(s["x"], s["weight"], s["rstd"], s["dy"], s["dx"], s["dweight"], s["workspace"], dh=s["dh"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if kind == "adamw":
        if "optimiser" not in s:      # the list of tensors, as a training program keeps it
            s["optimiser"] = K.AdamW([K.AdamWTensor(q["p"], q["g"], q["m"], q["v"], q["m_scale"], q["v_scale"], q["master"], q["decay"])
                                      for q in s["tensors"].values()], beta1=B1, beta2=B2, eps=ADAM_EPS, seed=SEED)
        s["optimiser"].step(s["t"], LR)
        s["t"] += 1
        return _adamw_outputs(s)
    if kind == "mx4_quantise":
        K.clt_mx4_quantise(s["a"], s["codes"], s["scales"], a_scale=s["a_scale"], transposed=case["transposed"])
        K.clt_mx4_dequantise(s["codes"], s["scales"], s["out"])
        return {"values": s["out"]}
    K.clt_mx4_quantise(s["x"], s["x_codes"], s["x_scales"])
    K.clt_mx4_product(s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["out"], case["d"], bias=s["bias"], theta=s["theta"])
    return {"z": s["out"]}


# ---- in 64 bits, from the definitions --------------------------------------------------------------------------------

def _nearest_4bit(x):
    """[..., K] double: per 32 elements the power of two that leaves no element off by more than half a step of 4-bit floats."""
    K = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, (32 - K % 32) % 32))
    x = x.view(*x.shape[:-1], -1, 32)
    mant, ex = torch.frexp(x.abs().amax(-1, keepdim=True))          # mant in [1/2, 1)
    ex = torch.where(mant >= 0.875, ex, ex - 1) - 2
    a = torch.ldexp(x, -ex.double())
    grid = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0)).double()
    return torch.ldexp(torch.round(a / grid) * grid, ex.double()).flatten(-2)[..., :K]


def _values_4bit(codes, scales, rows, K):
    """[L, rows, K] double out of the packed form, one 64-row panel and 128-element step after the other as 16 x 32 tiles."""
    L, rp, kp = scales.shape[:3]
    nibbles = torch.stack((codes.long() % 16, codes.long() // 16), -1).view(L, rp, 4, kp, 4, 16, 32)
    magnitude, exponent = nibbles % 2, nibbles // 2 % 4
    v = torch.where(exponent == 0, 0.5 * magnitude, torch.exp2(exponent.double() - 1) * (1 + 0.5 * magnitude)) * (1 - 2 * (nibbles // 8))
    e = scales.double().view(L, rp, kp, 4, 16, 4).permute(0, 1, 5, 2, 3, 4)      # layer, panel, 16 rows, step, block, row
    v = v * torch.exp2(e - 127)[..., None]
    return v.permute(0, 1, 2, 5, 3, 4, 6).reshape(L, rp * 64, kp * 128)[:, :rows, :K]


def _float8(x, uniform, mantissa, lowest_exponent):
    """Non-negative doubles -> 8-bit floats: the value's step, the part below it rounded up with the probability of its size."""
    _, ex = torch.frexp(x)
    step = torch.exp2((ex - 1).clamp_min(lowest_exponent).double() - mantissa)
    return torch.floor(x / step + uniform) * step


def _exact_adamw(q, index, t):
    eight = q["m_scale"] is not None
    shape, n = q["p"].shape, q["p"].numel()
    g, m, v = (q[k].reshape(-1) for k in "gmv")
    g = g.double()
    if eight:
        block = torch.arange(n, device=DEVICE) // 128
        m = m.view(torch.float8_e4m3fn).double() * torch.exp2(q["m_scale"].double() - 127)[block]
        v = v.view(torch.float8_e5m2).double() * torch.exp2(q["v_scale"].double() - 127)[block]
    m, v = m.double(), v.double()
    m, v = m + (1 - B1) * (g - m), v + (1 - B2) * (g * g - v)
    p = (q["p"] if q["master"] is None else q["master"]).double().reshape(-1)
    p = p - LR * q["decay"] * p - LR * (m / (1 - B1 ** t)) / (torch.sqrt(v / (1 - B2 ** t)) + ADAM_EPS)
    out = {"p": p.view(shape), "master": p.view(shape) if q["master"] is not None else None}
    del p, g
    if not eight:
        return dict(out, m=m.view(shape), v=v.view(shape), m_scale=None, v_scale=None)
    bits = _mix(torch.arange(n, device=DEVICE) ^ _key(t, index))

    def code(x, draw, mantissa, lowest):      # the element relative to its block's power of two, and that power
        top = torch.nn.functional.pad(x.abs(), (0, -n % 128)).view(-1, 128).amax(1)
        mant, ex = torch.frexp(top)
        ex = torch.where(mant > 0.875, ex, ex - 1) - (8 if mantissa == 3 else 15)
        return torch.sign(x) * _float8(torch.ldexp(x.abs(), -ex.double()[block]), (draw + 0.5) / 65536, mantissa, lowest), torch.exp2(ex.double())

    mc, ms = code(m, (bits % 65536).double(), 3, -6)
    vc, vs = code(v, (bits // 65536).double(), 2, -14)
    vc = torch.where(v > 0, vc.clamp_min(2.0 ** -16), vc)
    return dict(out, m=mc.view(shape), v=vc.view(shape), m_scale=ms, v_scale=vs)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = (h + s["residual"].double()).to(s["x"].dtype).double()
        rstd = 1.0 / torch.sqrt((h * h).sum(-1) / case["d"] + EPS)
        y = h * rstd[..., None] * s["weight"].double()[:, None, :]
        out = {"rstd": rstd, "h": h} if case["residual"] else {"rstd": rstd}
        if case["int8"]:
            out["scale"] = y.abs().amax(-1) / 127.0
            y = torch.round(y / out["scale"][..., None]) * out["scale"][..., None]
        return dict(out, y=y)
    if kind == "norm_backward":
        h, r, w, dy = s["x"].double(), s["rstd"].double()[..., None], s["weight"].double()[:, None, :], s["dy"].double()
        n = h * r      # normalised rows: dn = w dy, and the part of it along n does not reach h
        dn = w * dy
        dx = r * (dn - n * (dn * n).sum(-1, keepdim=True) / case["d"])
        return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dweight": (dy * n).sum(1)}
    if kind == "adamw":
        return {name: _exact_adamw(q, k, s["t"]) for k, (name, q) in enumerate(s["tensors"].items())}
    if kind == "mx4_quantise":
        a = s["a"].double()
        if s["a_scale"] is not None:
            a = (a * s["a_scale"].double()[..., None]).float().double()      # the product in 32 bits is the value that is cached
        return {"values": _nearest_4bit(a.mT.contiguous() if case["transposed"] else a)}
    x, w = _nearest_4bit(s["x"].double()), _values_4bit(s["w_codes"], s["w_scales"], case["F"], case["d"])
    pre = torch.stack([x[l] @ w[l].T.contiguous() for l in range(case["L"])]) + s["bias"].double()[:, None, :]
    return {"z": pre if s["theta"] is None else torch.where(pre > s["theta"].double()[:, None, :], pre, 0.0)}


def work(case):
    """Every input read once, every output written once."""
    L, B, d, F, kind = case["L"], case["B"], case["d"], case["F"], case["kind"]
    e = 2 if case["dtype"] == "bf16" else 4
    n = 1.0 * L * B * d
    if kind == "norm":
        bytes_ = n * e * (3 if case["residual"] else 1) + (n + 4.0 * L * B if case["int8"] else n * e) + 4.0 * L * (B + d)
        return {"bytes": bytes_, "flops": 6 * n}
    if kind == "norm_backward":
        return {"bytes": n * e * (4 if case["residual"] else 3) + 4.0 * L * (B + 2 * d), "flops": 10 * n}
    if kind == "adamw":
        matrices, vectors = (L * (L + 1) // 2 + L) * F * 1.0 * d, 2.0 * L * F + L * d
        state = 16.0 if case["states"] == 32 else 4.0 + 4.0 / 128
        return {"bytes": matrices * (3 * e + state + (8.0 if case["master"] else 0.0)) + vectors * 28.0, "flops": 12 * (matrices + vectors)}
    if kind == "mx4_quantise":      # rows to 4 bits (with a scale per 32), and back
        rows = F if case["transposed"] else B
        n = 1.0 * L * rows * d
        return {"bytes": n * (1 if case["int8"] else e) + 2 * n * 17 / 32 + n * e, "flops": 3 * n}
    return {"bytes": n * e + (n + 1.0 * L * F * d) * 17 / 32 + 1.0 * L * B * F * e + 8.0 * L * F, "flops": 2.0 * n * F}
