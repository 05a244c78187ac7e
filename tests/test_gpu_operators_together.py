"""The operators around the training step in one program, as they are used: residual streams through the RMS norm into int8 inputs,
training steps on them with AdamW and 8-bit moments, the trained encoder and the activations in 4 bits, features from their product."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as R
from operators_testlib import DEV, U, np32, np64

pytestmark = pytest.mark.gpu
L, B, d, F = 3, 260, 264, 520
MATRICES = ("W_enc", "W_dec")


def _program(K, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    params = {"W_enc": (n(L, d, F) / d ** 0.5).bfloat16(), "b_enc": 0.01 * n(L, F), "theta": torch.full((L, F), 0.03, device=DEV),
              "W_dec": (n(L * (L + 1) // 2, F, d) / d ** 0.5).bfloat16(), "b_dec": torch.zeros(L, d, device=DEV)}
    master = {k: params[k].float() for k in MATRICES}
    step = K.CLTStep(L, d, F, B, int8_inputs=True, master_weights=True, device=DEV)
    streams = [(n(L, B, d).bfloat16(), n(L, B, d).bfloat16(), n(L, B, d).bfloat16()) for _ in range(3)]
    weight = 1 + 0.1 * n(L, d)
    q, qs = torch.empty(L, B, d, dtype=torch.int8, device=DEV), torch.empty(L, B, device=DEV)
    y, ys = torch.empty_like(q), torch.empty_like(qs)
    h = torch.empty(L, B, d, dtype=torch.bfloat16, device=DEV)
    ones = torch.ones(L, d, device=DEV)
    return params, master, step, streams, weight, (q, qs), (y, ys), h, ones


def test_from_residual_streams_to_features_in_4_bits():
    from paper_2603_21014_amd import binding as K
    params, master, step, streams, weight, (q, qs), (y, ys), h, ones = _program(K)
    opt = step.adamw(params, bits=8, master=master, weight_decay=0.01, seed=77)
    names = list(step.grads)
    moments = lambda i: [None if a is None else a.cpu().numpy().copy() for a in opt.tensors[i].tensors[2:6]]
    state = {k: moments(i) for i, k in enumerate(names)}
    for t, (x, r, target) in enumerate(streams, 1):
        K.clt_rms_norm(x, weight, 1e-5, q=q, q_scale=qs, residual=r, h=h)
        K.clt_rms_norm(target, ones, 1e-5, q=y, q_scale=ys)
        step.train_step(q, y, params, None, None, t, 1e-3, 2.0, x_scale=qs, y_scale=ys, optimiser=opt)
        torch.cuda.synchronize()
        assert torch.isfinite(step.loss_dev).all()
        for i, k in enumerate(names):      # every moment is the oracle's, bit for bit, from the gradients that the step left
            m, v, ms, vs = state[k]
            matrix = k in MATRICES
            w = np32(master[k] if matrix else params[k]).reshape(-1)
            o = R.adamw(w, np32(step.grads[k]).reshape(-1), m.reshape(-1), v.reshape(-1), t, 1e-3, 0.9, 0.999, 1e-8, 0.01 if matrix else 0.0, ms, vs, 77, i)
            now = moments(i)
            assert np.array_equal(now[0].reshape(-1), o["m"]) and np.array_equal(now[1].reshape(-1), o["v"])
            if matrix:
                assert np.array_equal(now[2], o["m_scale"]) and np.array_equal(now[3], o["v_scale"])
                assert torch.equal(params[k], master[k].bfloat16())
            state[k] = now
    # the encoder in 4 bits on the last batch, from the int8 cache
    K.clt_rms_norm(streams[0][0], weight, 1e-5, q=q, q_scale=qs, residual=streams[0][1], h=h)
    step.forward(q, params, qs)
    wc, ws = K.mx4_empty(L, F, d)
    xc, xs = K.mx4_empty(L, B, d)
    K.clt_mx4_quantise(params["W_enc"], wc, ws, transposed=True)
    K.clt_mx4_quantise(q, xc, xs, a_scale=qs)
    z = torch.empty(L, B, F, dtype=torch.bfloat16, device=DEV)
    K.clt_mx4_product(xc, xs, wc, ws, z, d, bias=params["b_enc"], theta=params["theta"])
    xv = R.mx4_values(*R.mx4_round(np32(q) * np32(qs)[..., None]))[..., :d]
    wv = R.mx4_values(*R.mx4_round(np32(params["W_enc"]).transpose(0, 2, 1)))[..., :d]
    pre = np.matmul(xv, wv.transpose(0, 2, 1)) + np64(params["b_enc"])[:, None, :]
    err = (np.matmul(np.abs(xv), np.abs(wv).transpose(0, 2, 1)) + 1) * (d / 32 + 8) * U
    th, got = np64(params["theta"])[:, None, :], np64(z)
    near = np.abs(got - pre) <= err + np.abs(pre) * 2.0 ** -8 * 1.01
    assert np.all(np.where(pre > th + err, near, np.where(pre <= th - err, got == 0, near | (got == 0))))
    # and against the encoder on the unrounded operands: blocks are off by at most a quarter of their largest element's power of two
    # and about 0.08 of it in the mean square, d products of random signs: far closer than unrelated features would be
    full = np64(step.pre)
    assert np.linalg.norm(pre - full) < 0.3 * np.linalg.norm(full)


def test_a_program_captured_into_one_graph():
    """Norm, step, optimiser and 4-bit encoder as one graph, replayed, beside an eager twin of the same seeds."""
    from paper_2603_21014_amd import binding as K
    runs = []
    for captured in (False, True):
        params, master, step, streams, weight, (q, qs), (y, ys), h, ones = _program(K, seed=5)
        opt = step.adamw(params, bits=8, master=master, seed=3)
        wc, ws = K.mx4_empty(L, F, d)
        xc, xs = K.mx4_empty(L, B, d)
        z = torch.empty(L, B, F, dtype=torch.bfloat16, device=DEV)
        x, r, target = streams[0]

        def call():
            K.clt_rms_norm(x, weight, 1e-5, q=q, q_scale=qs, residual=r, h=h)
            K.clt_rms_norm(target, ones, 1e-5, q=y, q_scale=ys)
            step.train_step(q, y, params, None, None, 1, 1e-3, 2.0, x_scale=qs, y_scale=ys, optimiser=opt)
            K.clt_mx4_quantise(params["W_enc"], wc, ws, transposed=True)
            K.clt_mx4_quantise(q, xc, xs, a_scale=qs)
            K.clt_mx4_product(xc, xs, wc, ws, z, d, bias=params["b_enc"], theta=params["theta"])
        call()
        torch.cuda.synchronize()
        g = None
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call()
        seen = []
        for i in range(3):
            x.copy_(streams[i][0])      # other inputs at the same place
            g.replay() if captured else call()
            torch.cuda.synchronize()
            seen.append([z.clone(), params["W_dec"].clone(), q.clone(), opt.tensors[names(step).index("W_dec")].tensors[2].clone()])
        runs.append(seen)
    for a, b in zip(*runs):
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def names(step):
    return list(step.grads)


def test_adamw_asks_for_the_matrices_gradients():
    from paper_2603_21014_amd import binding as K
    step = K.CLTStep(L, d, F, B, device=DEV, matrix_grads=False)
    with pytest.raises(ValueError):
        step.adamw({})


def test_threshold_of_the_encoder_in_4_bits_is_that_of_the_step():
    """On operands that 4 bits hold exactly: the same features as clt_forward's, with the threshold held as its logarithm, and none of a token
    that is broken."""
    from paper_2603_21014_amd import binding as K
    g = torch.Generator().manual_seed(9)
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    some = lambda *s: values[torch.randint(0, 8, s, generator=g)] * (1 - 2 * torch.randint(0, 2, s, generator=g))
    x, w = some(L, B, d), some(L, d, F)
    x[:, :, ::32], w[:, ::32, :] = 6.0, -6.0      # (every block reaches the largest number, so that its scale is 1)
    x[1, 5, 40] = float("nan")
    params = {"W_enc": w.bfloat16().to(DEV), "b_enc": torch.zeros(L, F, device=DEV), "theta": torch.full((L, F), 4.5, device=DEV).log(),
              "W_dec": torch.zeros(L * (L + 1) // 2, F, d, dtype=torch.bfloat16, device=DEV), "b_dec": torch.zeros(L, d, device=DEV)}
    step = K.CLTStep(L, d, F, B, log_threshold=True, device=DEV)
    xd = x.bfloat16().to(DEV)
    step.forward(xd, params)
    wc, ws = K.mx4_empty(L, F, d)
    xc, xs = K.mx4_empty(L, B, d)
    K.clt_mx4_quantise(params["W_enc"], wc, ws, transposed=True)
    K.clt_mx4_quantise(xd, xc, xs)
    z = torch.empty(L, B, F, dtype=torch.bfloat16, device=DEV)
    K.clt_mx4_product(xc, xs, wc, ws, z, d, theta=params["theta"].exp())
    # (products are multiples of 1/4 and sums below 2^14: exact in fp32, and none is at the threshold's rounding)
    assert torch.equal(z, step.z) and (z != 0).any() and not torch.isnan(z).any()
    assert not z[1, 5].any() and xs.eq(255).any()
