"""A training step of a small recurrent language model through the library's operators, as a program would run it: gates and inputs
from one product, the recurrence, logits, log probabilities with an entropy term, the gradients back, and AdamW; against the
same in 64 bits."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import operator_forms as F
import paper_2008_11421_amd as K


def test_a_step_of_a_recurrent_model():
    import torch
    import gpu_util as g
    lib, rng = K.lib(), np.random.default_rng(31)
    T, D, V, starts = 700, 64, 520, [0, 130, 131, 500, 688]
    S, n = len(starts) - 1, starts[-1]
    bf = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).cuda()
    h64 = lambda t: t.float().cpu().numpy().astype(np.float64)
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    f32 = lambda *s: torch.zeros(s, device="cuda")
    x, wg, wo = bf(rng.standard_normal((T, D))), bf(rng.standard_normal((2 * D, D)) * 0.2), bf(rng.standard_normal((V, D)) * 0.3)
    tokens = torch.tensor(rng.integers(0, V, T), dtype=torch.int32, device="cuda")
    tokens[n:] = -1
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    q, none = g.stream_ptr(), None
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    W, size, u64 = g.ptr(ws), C.c_uint64(ws.numel()), C.c_uint64
    both, h, logits, dl, dh, dboth, dx = new(T, 2 * D), new(T, D), new(T, V), new(T, V), new(T, D), new(T, 2 * D), new(T, D)
    marks, lp, ent, stats, dwg, dwo = f32(3, D), f32(T), f32(T), f32(T, 2), f32(2 * D, D), f32(V, D)
    shape = K.ScanShape(tokens=T, channels=D, sequences=S, ld_gate=2 * D, ld_x=2 * D, ld_dgate=2 * D, ld_dx=2 * D)
    right = lambda t: C.c_void_p(t.data_ptr() + 2 * D)
    call = lambda status: (_ for _ in ()).throw(AssertionError(status)) if status else None
    call(lib.karma_k_gemm_bf16(g.ptr(x), g.ptr(wg), g.ptr(both), none, none, T, 2 * D, D, 0, W, size, q))
    call(lib.karma_k_gated_scan_fwd_bf16(g.ptr(both), right(both), none, g.ptr(st), g.ptr(h), none, g.ptr(marks), C.byref(shape), W, size, q))
    call(lib.karma_k_gemm_bf16(g.ptr(h), g.ptr(wo), g.ptr(logits), none, none, T, V, D, 0, W, size, q))
    call(lib.karma_k_token_logprob_fwd_bf16(g.ptr(logits), u64(0), g.ptr(tokens), g.ptr(lp), g.ptr(ent), g.ptr(stats), none, none, T, V, 0,
                                            C.c_float(1.0), W, size, q))
    up, ue = torch.full((T,), -1.0 / n, device="cuda"), torch.full((T,), -0.1 / n, device="cuda")       # loss: -mean(logprob + 0.1 entropy)
    ue[n:] = 0
    call(lib.karma_k_token_logprob_bwd_bf16(g.ptr(logits), u64(0), g.ptr(tokens), g.ptr(stats), g.ptr(ent), g.ptr(up), g.ptr(ue), g.ptr(dl), u64(0),
                                            T, V, C.c_float(1.0), q))
    call(lib.karma_k_gemm_bf16(g.ptr(dl), g.ptr(wo), g.ptr(dh), none, none, T, D, V, K.GEMM_B_STRIDED, W, size, q))
    call(lib.karma_k_gemm_bf16(g.ptr(dl), g.ptr(h), g.ptr(dwo), none, none, V, D, n, K.GEMM_A_STRIDED | K.GEMM_B_STRIDED | K.GEMM_OUT_F32, W, size, q))
    call(lib.karma_k_gated_scan_bwd_bf16(g.ptr(both), right(both), none, g.ptr(st), g.ptr(marks), g.ptr(dh), none, g.ptr(dboth), right(dboth), none,
                                         C.byref(shape), W, size, q))
    call(lib.karma_k_gemm_bf16(g.ptr(dboth), g.ptr(wg), g.ptr(dx), none, none, T, D, 2 * D, K.GEMM_B_STRIDED, W, size, q))
    call(lib.karma_k_gemm_bf16(g.ptr(dboth), g.ptr(x), g.ptr(dwg), none, none, 2 * D, D, n, K.GEMM_A_STRIDED | K.GEMM_B_STRIDED | K.GEMM_OUT_F32,
                               W, size, q))
    torch.cuda.synchronize()

    # the same in 64 bits, from the same bf16 inputs
    x6, wg6, wo6, tok = h64(x), h64(wg), h64(wo), tokens.cpu().numpy()
    b6 = x6 @ wg6.T
    hh, _, _ = F.scan_forward(b6[:, :D], b6[:, D:], starts)
    z = hh @ wo6.T
    r = F.logprob_forward(z, tok, 1.0)
    loss = -(r["logprob"][:n] + 0.1 * r["entropy"][:n]).mean()
    dz = F.logprob_backward(z, tok, 1.0, np.full(T, -1.0 / n), np.where(np.arange(T) < n, -0.1 / n, 0.0))
    dh6 = dz @ wo6
    dg6, dx6, _, _ = F.scan_backward(b6[:, :D], b6[:, D:], starts, dh6)
    db6 = np.concatenate([dg6, dx6], 1)
    got = -(lp[:n] + 0.1 * ent[:n]).double().mean().item()
    # every tensor between the operators is bf16: half a step, 2^-8 of an element, uncorrelated over the sums; the workload's bar is 2e-2
    assert abs(got - loss) <= 2e-3 * abs(loss)
    assert (dboth[n:] == 0).all() and (h[n:] == 0).all()
    for a, b in ((h[:n], hh[:n]), (dl, dz), (dboth, db6), (dx, db6 @ wg6), (dwo, dz[:n].T @ hh[:n]), (dwg, db6[:n].T @ x6[:n])):
        assert g.rel_l2(h64(a), b) <= 2e-2

    # and the update of both weights, states in 8 and in 32 bits
    master = [t.float().clone() for t in (wg, wo)]
    before = [t.clone() for t in master]
    m, v = [torch.zeros(wg.numel(), dtype=torch.int8, device="cuda"), f32(V * D)], [torch.zeros(wg.numel(), dtype=torch.uint8, device="cuda"), f32(V * D)]
    sc = [f32(wg.numel() // 64), f32(wg.numel() // 64)]
    ts = (K.AdamwTensor * 2)(
        K.AdamwTensor(w=master[0].data_ptr(), m=m[0].data_ptr(), v=v[0].data_ptr(), m_scale=sc[0].data_ptr(), v_scale=sc[1].data_ptr(),
                      grad=dwg.data_ptr(), out=wg.data_ptr(), n=wg.numel(), weight_decay=0.1, flags=K.ADAMW_OUT_BF16 | K.ADAMW_STATES_8BIT),
        K.AdamwTensor(w=master[1].data_ptr(), m=m[1].data_ptr(), v=v[1].data_ptr(), grad=dwo.data_ptr(), out=wo.data_ptr(), n=wo.numel(),
                      weight_decay=0.1, flags=K.ADAMW_OUT_BF16))
    now = K.AdamwStep(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=1.0, seed=1, step=1)
    call(lib.karma_k_adamw(ts, 2, C.byref(now), none, q))
    torch.cuda.synchronize()
    for w0, w1, gr, low in zip(before, master, (dwg, dwo), (wg, wo)):
        want, _, _ = F.adamw(w0.cpu().numpy(), np.zeros(w0.shape), np.zeros(w0.shape), gr.cpu().numpy(), 0.1, 1e-3, 0.9, 0.95, 1e-8, 1.0, 1)
        # |w| < 2 and the update is 1e-3: a few roundings of each
        assert np.abs(w1.cpu().numpy() - want).max() <= 8 * F.U * 2
        assert torch.equal(low, w1.to(torch.bfloat16).view_as(low))
