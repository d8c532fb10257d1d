"""A training step of an attention layer with normalised, rotated queries and keys through the library's operators, as a program would run it: the
projection, norms and rotation, attention, logits and their loss, the gradients back, the norm of them all and the clipped update; then the next
tokens from the logits; against the same in 64 bits."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import decoder_forms as D
import operator_forms as F
import paper_2008_11421_amd as K

B, S, H, d, V, EPS = 2, 128, 2, 64, 520, 1e-5
T, h = B * S, H * d


def attention(q, k, v):
    """(context, probabilities), [B][S][H][d], causal"""
    s = np.einsum("bihd,bjhd->bhij", q, k) / np.sqrt(d)
    s = np.where(np.tril(np.ones((S, S), bool)), s, -np.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return np.einsum("bhij,bjhd->bihd", p, v), p


def attention_back(q, k, v, p, dc):
    dv = np.einsum("bhij,bihd->bjhd", p, dc)
    dp = np.einsum("bihd,bjhd->bhij", dc, v)
    ds = p * (dp - (dp * p).sum(-1, keepdims=True)) / np.sqrt(d)
    return np.einsum("bhij,bjhd->bihd", ds, k), np.einsum("bhij,bihd->bjhd", ds, q), dv


@pytest.mark.parametrize("pairs", [False, True])
def test_a_step_of_an_attention_layer(pairs):
    import torch
    import gpu_util as g
    lib, rng = K.lib(), np.random.default_rng(41)
    bf = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).cuda()
    h64 = lambda t: t.float().cpu().numpy().astype(np.float64)
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    f32 = lambda *s: torch.zeros(s, device="cuda")
    x, wq, wo = bf(rng.standard_normal((T, h))), bf(rng.standard_normal((3 * h, h)) * 0.1), bf(rng.standard_normal((V, h)) * 0.3)
    gamma = [bf(1 + 0.2 * rng.standard_normal(d)) for _ in range(2)]
    freq = 10000.0 ** (-np.arange(d // 2) * 2 / d)
    tokens = torch.tensor(rng.integers(0, V, T), dtype=torch.int32, device="cuda")
    fr = torch.from_numpy(freq).cuda()
    q, none, u64 = g.stream_ptr(), None, C.c_uint64
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    W, size = g.ptr(ws), u64(ws.numel())
    raw, qkv, ctx, logits, dl, dctx, dqkv = new(T, 3 * h), new(T, 3 * h), new(T, h), new(T, V), new(T, V), new(T, h), new(T, 3 * h)
    lse, delta, lp, stats = f32(B, H, S), f32(B, H, S), f32(T), f32(T, 2)
    dwq, dwo, dg = f32(3 * h, h), f32(V, h), [f32(d), f32(d)]
    part = lambda t, k: C.c_void_p(t.data_ptr() + 2 * k * h)
    parts = lambda t: (part(t, 0), part(t, 1), part(t, 2))
    shape = K.QkShape(tokens=T, seq=S, heads_q=H, heads_k=H, heads_v=H, d=d, rot=d, flags=K.QK_NORM | (K.QK_PAIRS if pairs else 0), eps=EPS,
                      **{"ld_" + n: 3 * h for n in ("q", "k", "v", "yq", "yk", "yv", "dq", "dk", "dv")})

    def call(status):
        assert status == 0

    call(lib.karma_k_gemm_bf16(g.ptr(x), g.ptr(wq), g.ptr(raw), none, none, T, 3 * h, h, 0, W, size, q))
    call(lib.karma_k_qk_rotary_fwd_bf16(*parts(raw), g.ptr(gamma[0]), g.ptr(gamma[1]), none, g.ptr(fr), *parts(qkv), C.byref(shape), q))
    call(lib.karma_k_attention_fwd_bf16(g.ptr(qkv), g.ptr(ctx), g.ptr(lse), B, S, H, d, q))
    call(lib.karma_k_gemm_bf16(g.ptr(ctx), g.ptr(wo), g.ptr(logits), none, none, T, V, h, 0, W, size, q))
    call(lib.karma_k_token_logprob_fwd_bf16(g.ptr(logits), u64(0), g.ptr(tokens), g.ptr(lp), none, g.ptr(stats), none, none, T, V, 0, C.c_float(1.0), W, size, q))
    up = torch.full((T,), -1.0, device="cuda")
    call(lib.karma_k_token_logprob_bwd_bf16(g.ptr(logits), u64(0), g.ptr(tokens), g.ptr(stats), none, g.ptr(up), none, g.ptr(dl), u64(0), T, V, C.c_float(1.0), q))
    call(lib.karma_k_gemm_bf16(g.ptr(dl), g.ptr(wo), g.ptr(dctx), none, none, T, h, V, K.GEMM_B_STRIDED, W, size, q))
    strided = K.GEMM_A_STRIDED | K.GEMM_B_STRIDED | K.GEMM_OUT_F32
    call(lib.karma_k_gemm_bf16(g.ptr(dl), g.ptr(ctx), g.ptr(dwo), none, none, V, h, T, strided, W, size, q))
    call(lib.karma_k_attention_bwd_bf16(g.ptr(qkv), g.ptr(ctx), g.ptr(dctx), g.ptr(lse), g.ptr(delta), g.ptr(dqkv), B, S, H, d, q))
    # in place: the values' gradient is where it belongs
    call(lib.karma_k_qk_rotary_bwd_bf16(*parts(dqkv), part(raw, 0), part(raw, 1), g.ptr(gamma[0]), g.ptr(gamma[1]), none, g.ptr(fr), *parts(dqkv),
                                        g.ptr(dg[0]), g.ptr(dg[1]), C.byref(shape), W, size, q))
    call(lib.karma_k_gemm_bf16(g.ptr(dqkv), g.ptr(x), g.ptr(dwq), none, none, 3 * h, h, T, strided, W, size, q))
    grads = [dwq, dwo, *dg]
    gt = (K.GradTensor * 4)(*[K.GradTensor(grad=t.data_ptr(), n=t.numel()) for t in grads])
    live, norm = f32(4), f32(1)
    live[0] = 1e-3
    live.view(torch.int32)[2] = 1
    call(lib.karma_k_grad_norm(gt, 4, C.c_float(1.0), C.c_float(1.0 / T), g.ptr(norm), none, C.c_void_p(live.data_ptr() + 4), W, size, q))
    master = [t.float().clone() for t in (wq, wo, *gamma)]
    before = [t.clone() for t in master]
    m, v = [torch.zeros_like(t) for t in master], [torch.zeros_like(t) for t in master]
    ts = (K.AdamwTensor * 4)(*[K.AdamwTensor(w=w.data_ptr(), m=a.data_ptr(), v=b.data_ptr(), grad=gr.data_ptr(), n=w.numel())
                               for w, a, b, gr in zip(master, m, v, grads)])
    now = K.AdamwStep(lr=0, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=0, seed=0, step=1)
    call(lib.karma_k_adamw(ts, 4, C.byref(now), g.ptr(live), q))
    rule = torch.tensor([[0.8, 0.9, 0.0, 0.0]], device="cuda")
    rule.view(torch.int32)[0, 3] = 40
    uniform = torch.from_numpy(rng.random(T).astype(np.float32)).cuda()
    drawn, drawn_lp, kept = torch.zeros(T, dtype=torch.int32, device="cuda"), f32(T), torch.zeros(T, dtype=torch.int32, device="cuda")
    call(lib.karma_k_sample_bf16(g.ptr(logits), u64(0), g.ptr(rule), 1, g.ptr(uniform), g.ptr(drawn), g.ptr(drawn_lp), g.ptr(kept), T, V, W, size, q))
    torch.cuda.synchronize()

    # the same in 64 bits, from the same bf16 inputs
    x6, wq6, wo6, g6, tok = h64(x), h64(wq), h64(wo), [h64(t) for t in gamma], tokens.cpu().numpy()
    raw6 = x6 @ wq6.T
    third = lambda a, k: a[:, k * h:(k + 1) * h].reshape(T, H, d)
    angle = (np.arange(T) % S)[:, None] * freq
    q6, k6 = (D.qk_forward(third(raw6, k), g6[k], angle, d, pairs, EPS)[0].reshape(B, S, H, d) for k in range(2))
    v6 = third(raw6, 2).reshape(B, S, H, d)
    c6, p6 = attention(q6, k6, v6)
    c6 = c6.reshape(T, h)
    z = c6 @ wo6.T
    r = F.logprob_forward(z, tok, 1.0)
    dz = F.logprob_backward(z, tok, 1.0, np.full(T, -1.0))
    dq6, dk6, dv6 = attention_back(q6, k6, v6, p6, (dz @ wo6).reshape(B, S, H, d))
    (dq6, dgq, _, _), (dk6, dgk, _, _) = (D.qk_backward(a.reshape(T, H, d), third(raw6, k), g6[k], angle, d, pairs, EPS) for k, a in enumerate((dq6, dk6)))
    draw6 = np.concatenate([dq6.reshape(T, h), dk6.reshape(T, h), dv6.reshape(T, h)], 1)
    grads6 = [draw6.T @ x6, dz.T @ c6, dgq, dgk]
    # every tensor between the operators is bf16: half a step, 2^-8 of an element, uncorrelated over the sums; attention's own bars are 2^-6
    # forward and 2^-4 backward
    assert g.rel_l2(h64(qkv[:, :2 * h]), np.concatenate([q6.reshape(T, h), k6.reshape(T, h)], 1)) <= 2e-2
    assert g.rel_l2(h64(ctx), c6) <= 2.0 ** -6 and g.rel_l2(h64(logits), z) <= 2e-2
    assert abs(lp.double().mean().item() - r["logprob"].mean()) <= 1e-2 * abs(r["logprob"].mean())
    assert g.rel_l2(h64(dl), dz) <= 2e-2 and g.rel_l2(h64(dwo), grads6[1]) <= 2e-2
    assert g.rel_l2(h64(dqkv), draw6) <= 2.0 ** -4
    for a, b in zip((dwq, *dg), (grads6[0], *grads6[2:])):
        assert g.rel_l2(h64(a), b) <= 2.0 ** -4
    # the norm is that of these gradients, and the update that of the clipped ones
    want, factor, _ = D.grad_norm([h64(t) for t in grads], 1.0, 1.0 / T)
    assert abs(norm.item() - want) <= 2 * D.U * want and abs(live[1].item() - factor) <= 2 * D.U * factor
    assert g.rel_l2([want], [np.sqrt(sum((t ** 2).sum() for t in grads6)) / T]) <= 2.0 ** -4
    for w0, w1, gr in zip(before, master, grads):
        w6, _, _ = F.adamw(w0.cpu().numpy(), np.zeros(w0.shape), np.zeros(w0.shape), gr.cpu().numpy(), 0.0, 1e-3, 0.9, 0.95, 1e-8, live[1].item(), 1)
        # |w| < 2 and the update is 1e-3: a few roundings of each
        assert np.abs(w1.cpu().numpy() - w6).max() <= 8 * D.U * 2
    # the tokens drawn are those of these logits
    zl, u = h64(logits), uniform.cpu().numpy()
    for t in range(T):
        token, logprob, n = D.sample_row(zl[t], np.float32(0.8), np.float32(0.9), 0.0, 40, u[t])
        assert (drawn[t].item(), kept[t].item()) == (token, n) and abs(drawn_lp[t].item() - logprob) <= D.U * abs(logprob) + 1e-9
