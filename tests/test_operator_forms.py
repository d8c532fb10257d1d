"""The plain forms of the recurrence, the log probabilities and the AdamW step: gradients against central differences, closed
forms, and what the entry points refuse (no GPU is needed for a refusal)."""
import ctypes as C

import numpy as np
import pytest

import operator_forms as F
import paper_2008_11421_amd as K


def test_scan_gradients_against_differences():
    rng = np.random.default_rng(1)
    starts = [0, 3, 3, 9]
    f, x, dh = (rng.standard_normal((9, 2)) for _ in range(3))
    h0, dl = rng.standard_normal((3, 2)), rng.standard_normal((3, 2))

    def loss(f, x, h0):
        h, _, last = F.scan_forward(f, x, starts, h0)
        return (h * dh).sum() + (last * dl).sum()

    dgate, dx, dh0, _ = F.scan_backward(f, x, starts, dh, h0, dl)
    for k, (a, got) in enumerate(((f, dgate), (x, dx), (h0, dh0))):
        want = np.zeros_like(a)
        for i in np.ndindex(a.shape):
            args = [f.copy(), x.copy(), h0.copy()]
            args[k][i] += 1e-5
            up = loss(*args)
            args[k][i] -= 2e-5
            want[i] = (up - loss(*args)) / 2e-5
        # the differences are off by h^2 / 6 times the third derivative (about 1) and 1e-16 / h
        assert np.abs(got - want).max() < 1e-8, k
    assert np.array_equal(dh0[1], dl[1])        # a sequence without tokens hands its gradient on


def test_scan_closed_forms():
    x = np.full((200, 1), 3.0)
    f = np.full((200, 1), 2.0)
    h, _, _ = F.scan_forward(f, x, [0, 200])
    a = 1 / (1 + np.exp(-2.0))
    assert np.allclose(h[:, 0], 3.0 * (1 - a ** np.arange(1, 201)), rtol=0, atol=1e-13)


def scan_in_fp32(f, x, dh, h0, dh_last, by_sign):
    """One sequence in fp32, step by step: the share b rounded by itself and 1 - b taken from it, or (by_sign) the smaller share of the two."""
    w = np.float32
    f, x, dh = (np.asarray(a, w) for a in (f, x, dh))
    E = np.exp(-np.abs(f) if by_sign else f)
    small = E / (w(1) + E)
    neg = f < 0
    b = w(1) / (w(1) + E)
    h, states, g, out = np.asarray(h0, w), [], np.asarray(dh_last, w), dict(h=[], dgate=[], dx=[])
    for t in range(len(f)):
        states.append(h)
        if by_sign:
            h = np.where(neg[t], x[t] + small[t] * (h - x[t]), h + small[t] * (x[t] - h))
        else:
            h = h + b[t] * (x[t] - h)
        out["h"].append(h)
    last = h
    for t in range(len(f) - 1, -1, -1):
        D, gap = dh[t] + g, states[t] - x[t]
        if by_sign:
            s = small[t]
            ab, dx, g = s - s * s, np.where(neg[t], D - s * D, s * D), np.where(neg[t], s * D, D - s * D)
        else:
            ab, dx = b[t] - b[t] * b[t], b[t] * D
            g = D - dx
        out["dgate"].insert(0, D * gap * ab)
        out["dx"].insert(0, dx)
    return {**{k: np.array(v) for k, v in out.items()}, "h_last": last[None], "dh0": g[None]}


@pytest.mark.parametrize("bias", [-30.0, -16.0, -10.0, 0.0, 3.0, 12.0])
def test_scan_bounds_tell_where_bits_are_lost(bias):
    """fp32 arithmetic with the smaller of the two shares stays within the bounds whatever the gates; with one minus the other share it does
    not where gates are clearly negative."""
    rng = np.random.default_rng(int(bias) + 100)
    f, x, dh = (rng.standard_normal((400, 6)).astype(np.float32) for _ in range(3))
    f += np.float32(bias)
    h0, dl = (rng.standard_normal((1, 6)).astype(np.float32) for _ in range(2))
    h0[0, :3] *= 1e8
    want, bound = F.scan_by_shares(f, x, [0, 400], h0, dh, dl)
    far = lambda got: {k: float((np.abs(got[k].astype(np.float64) - want[k]) / (bound[k] + 1e-300)).max()) for k in want}
    assert max(far(scan_in_fp32(f, x, dh, h0[0], dl[0], True)).values()) <= 1
    by_b = far(scan_in_fp32(f, x, dh, h0[0], dl[0], False))
    if bias <= -10:
        assert by_b["dgate"] > 10 and by_b["dh0"] > 10 and by_b["h"] > 10


def test_scan_by_shares_is_the_scan():
    rng = np.random.default_rng(4)
    starts = [0, 3, 3, 9]
    f, x, dh = (rng.standard_normal((9, 2)) for _ in range(3))
    h0, dl = rng.standard_normal((3, 2)), rng.standard_normal((3, 2))
    got, _ = F.scan_by_shares(f, x, starts, h0, dh, dl)
    h, _, last = F.scan_forward(f, x, starts, h0)
    dgate, dx, dh0, _ = F.scan_backward(f, x, starts, dh, h0, dl)
    for k, want in dict(h=h, h_last=last, dgate=dgate, dx=dx, dh0=dh0).items():
        assert np.abs(got[k] - want).max() < 1e-14, k


def test_logprob_gradients_against_differences():
    rng = np.random.default_rng(2)
    z, tokens = rng.standard_normal((4, 7)), np.array([3, -1, 0, 6])
    z[2, 5] = -np.inf
    dl, de = rng.standard_normal(4), rng.standard_normal(4)
    loss = lambda z: (lambda r: (r["logprob"] * dl).sum() + (r["entropy"] * de).sum())(F.logprob_forward(z, tokens, 1.3))
    got = F.logprob_backward(z, tokens, 1.3, dl, de)
    for i in np.ndindex(z.shape):
        if z[i] > -np.inf:
            up, dn = z.copy(), z.copy()
            up[i] += 1e-5
            dn[i] -= 1e-5
            assert abs(got[i] - (loss(up) - loss(dn)) / 2e-5) < 1e-8, i
        else:
            assert got[i] == 0


def test_logprob_closed_forms():
    r = F.logprob_forward(np.zeros((1, 8)), np.array([2]), 0.5, 3)
    assert np.allclose(r["logprob"], -np.log(8)) and np.allclose(r["entropy"], np.log(8)) and r["top_id"].tolist() == [[0, 1, 2]]
    r = F.logprob_forward(np.full((1, 4), -np.inf), np.array([2]), 1.0, 2)
    assert r["logprob"][0] == -np.inf and r["entropy"][0] == 0 and r["top_id"].tolist() == [[0, 1]]


def test_adamw_first_step_is_the_sign():
    w, m, v = F.adamw(np.ones(3), np.zeros(3), np.zeros(3), np.array([2.0, -0.5, 0.0]), 0.1, 0.01, 0.9, 0.95, 1e-12, 1.0, 1)
    assert np.allclose(w, 1 - F.f32(0.01) * F.f32(0.1) - F.f32(0.01) * np.array([1, -1, 0]), atol=1e-10)


def test_codes_keep_the_expectation():
    """Over 512 seeds the mean of the values that the codes stand for is the value, within six deviations of the mean."""
    rng = np.random.default_rng(3)
    m, v = rng.standard_normal(256) * 1e-3, rng.standard_normal(256) ** 2 * 1e-6
    ms, vs = [], []
    for seed in range(512):
        cm, sm, cv, sv = F.quantised(m, v, 5, seed)
        ms.append(cm * F.by_block(sm, 256))
        vs.append(cv.astype(float) ** 2 * F.by_block(sv, 256))
    ms, vs = np.array(ms), np.array(vs)
    assert (np.abs(ms.mean(0) - m) <= 6 * F.by_block(sm, 256) * 0.5 / np.sqrt(512)).all()
    step = (2 * np.sqrt(v / F.by_block(sv, 256)) + 1) * F.by_block(sv, 256)
    far = v >= F.by_block(sv, 256)      # below one code a value is held up on purpose
    assert far.sum() > 200 and (np.abs(vs.mean(0) - v)[far] <= 6 * (step * 0.5 / np.sqrt(512))[far]).all()
    assert (vs > 0).all()


# ------------------------------------------------------------------------------------------------- refusals
P = C.c_void_p(4096)        # a pointer that no call here may follow


def scan_fwd(shape, gate=P, x=P, h=P, starts=None, ws=P, ws_bytes=1 << 40, fn=None):
    return (fn or K.lib().karma_k_gated_scan_fwd_bf16)(gate, x, None, starts, h, None, None, C.byref(shape) if shape else None, ws, C.c_uint64(ws_bytes), None)


def test_scan_refusals():
    good = dict(tokens=512, channels=8, sequences=2)
    S = lambda **k: K.ScanShape(**{**good, **k})
    assert scan_fwd(None) == K.E_INVAL
    for bad in (dict(channels=0), dict(sequences=0), dict(tokens=511), dict(tokens=(1 << 31) - 1024), dict(ld_gate=7), dict(ld_x=4), dict(ld_h=1),
                dict(ld_dx=7), dict(channels=1 << 31), dict(ld_gate=1 << 62)):
        assert scan_fwd(S(**bad)) == K.E_INVAL, bad
        assert K.gated_scan_ws_bytes(S(**bad)) == 0 or bad == dict(tokens=511), bad
    for missing in ("gate", "x", "h"):
        assert scan_fwd(S(), **{missing: None}) == K.E_INVAL, missing
        assert scan_fwd(S(), **{missing: C.c_void_p(4097)}) == K.E_INVAL, missing
        assert scan_fwd(S(), fn=K.lib().karma_k_gated_scan_fwd_f32, **{missing: C.c_void_p(4098)}) == K.E_INVAL, missing
    args = dict(gate=P, x=P, marks=P, dh=P, dgate=P, dx=P)
    for missing in args:
        a = dict(args, **{missing: None})
        assert K.lib().karma_k_gated_scan_bwd_bf16(a["gate"], a["x"], None, None, a["marks"], a["dh"], None, a["dgate"], a["dx"], None,
                                                   C.byref(S()), P, C.c_uint64(1 << 40), None) == K.E_INVAL, missing


def logprob_fwd(rows=4, cols=100, ld=0, top=0, scale=1.0, logits=P, tokens=P, logprob=P, entropy=None, stats=None, top_lp=None, top_id=None,
                fn="bf16", ws=P, ws_bytes=1 << 40):
    return getattr(K.lib(), "karma_k_token_logprob_fwd_" + fn)(logits, C.c_uint64(ld), tokens, logprob, entropy, stats, top_lp, top_id, C.c_uint32(rows),
                                                               C.c_uint32(cols), C.c_uint32(top), C.c_float(scale), ws, C.c_uint64(ws_bytes), None)


def logprob_bwd(rows=4, cols=100, ld=0, ld_d=0, scale=1.0, logits=P, tokens=P, stats=P, entropy=P, dl=P, de=P, out=P, fn="bf16"):
    return getattr(K.lib(), "karma_k_token_logprob_bwd_" + fn)(logits, C.c_uint64(ld), tokens, stats, entropy, dl, de, out, C.c_uint64(ld_d),
                                                               C.c_uint32(rows), C.c_uint32(cols), C.c_float(scale), None)


def test_logprob_refusals():
    for bad in (dict(cols=0), dict(ld=99), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e21), dict(scale=1e-21), dict(tokens=None),
                dict(logprob=None), dict(top=2), dict(top=2, top_lp=P), dict(top=65, top_lp=P, top_id=P), dict(cols=3, top=4, top_lp=P, top_id=P),
                dict(logits=None), dict(logits=C.c_void_p(4097)), dict(logits=C.c_void_p(4098), fn="f32"), dict(rows=1 << 31), dict(ld=1 << 62),
                dict(cols=1 << 31)):
        assert logprob_fwd(**bad) == K.E_INVAL, bad
    for bad in (dict(cols=0), dict(ld=99), dict(ld_d=99), dict(scale=0.0), dict(tokens=None), dict(entropy=None), dict(dl=None, de=None), dict(stats=None),
                dict(out=None), dict(out=C.c_void_p(4097)), dict(out=C.c_void_p(4098), fn="f32"), dict(logits=None)):
        assert logprob_bwd(**bad) == K.E_INVAL, bad
    assert logprob_fwd(rows=0, logits=None) == K.OK and logprob_bwd(rows=0, logits=None, out=None, stats=None) == K.OK


def test_adamw_refusals():
    now = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=1.0, seed=1, step=1)
    tensor = dict(w=4096, m=4096, v=4096, grad=4096, n=10, flags=0)

    def call(now_change=None, live=None, **change):
        t = (K.AdamwTensor * 1)(K.AdamwTensor(**{**tensor, **change}))
        return K.lib().karma_k_adamw(t, 1, C.byref(K.AdamwStep(**{**now, **(now_change or {})})), live, None)

    lib = K.lib()
    assert lib.karma_k_adamw(None, 0, None, None, None) == K.E_INVAL
    assert lib.karma_k_adamw(None, 1, C.byref(K.AdamwStep(**now)), None, None) == K.E_INVAL
    assert lib.karma_k_adamw(None, 0, C.byref(K.AdamwStep(**now)), None, None) == K.OK
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=-1.0)):
        assert call(bad) == K.E_INVAL, bad
    for bad in (dict(w=None), dict(m=None), dict(v=None), dict(grad=None), dict(w=4098), dict(grad=4098), dict(grad=4097, flags=1), dict(out=4098),
                dict(out=4097, flags=2), dict(flags=4), dict(flags=4, m_scale=4096), dict(flags=8), dict(m=4098), dict(n=1 << 50),
                dict(flags=4, m_scale=4096, v_scale=4098)):
        assert call(**bad) == K.E_INVAL, bad
    assert call(live=C.c_void_p(4098)) == K.E_INVAL
    assert call(n=0, w=None, m=None, v=None, grad=None) == K.OK
    ptrs = (C.c_void_p * 1)(4096)
    t = (K.AdamwTensor * 1)(K.AdamwTensor(**tensor))
    assert lib.karma_k_adamw_states(t, 1, ptrs, ptrs, None) == K.E_INVAL            # fp32 states
    t = (K.AdamwTensor * 1)(K.AdamwTensor(**dict(tensor, flags=4, m_scale=4096, v_scale=4096)))
    assert lib.karma_k_adamw_states(t, 1, (C.c_void_p * 1)(None), ptrs, None) == K.E_INVAL
    assert lib.karma_k_adamw_states(t, 1, None, ptrs, None) == K.E_INVAL


def test_sizes_beyond_a_launch_are_refused():
    for bad in (dict(tokens=1 << 30, channels=64, sequences=1), dict(tokens=(1 << 31) - 2048, channels=1, sequences=1),
                dict(tokens=1 << 26, channels=1, sequences=1 << 26), dict(tokens=1024, channels=1 << 27, sequences=2)):
        assert scan_fwd(K.ScanShape(**bad), ws_bytes=1 << 62) == K.E_INVAL and K.gated_scan_ws_bytes(K.ScanShape(**bad)) == 0, bad
    assert K.gated_scan_ws_bytes(K.ScanShape(tokens=1 << 29, channels=64, sequences=1)) > 0
    assert logprob_fwd(rows=1 << 24, cols=4096) == K.E_INVAL and logprob_fwd(rows=1 << 26, cols=8) == K.E_INVAL
    assert logprob_bwd(rows=1 << 24, cols=8192) == K.E_INVAL and logprob_bwd(rows=1 << 26, cols=8) == K.E_INVAL
    step = K.AdamwStep(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=1.0, seed=1, step=1)
    t = (K.AdamwTensor * 1)(K.AdamwTensor(w=4096, m=4096, v=4096, grad=4096, n=1 << 34, flags=0))
    assert K.lib().karma_k_adamw(t, 1, C.byref(step), None, None) == K.E_INVAL


@pytest.mark.parametrize("odd", [1, 2, 3])
def test_operands_of_32_bits_off_their_boundaries_are_refused(odd):
    """The starts and states of a scan, the tokens, statistics and results of log probabilities: a scalar load drops an address's lowest bits."""
    Q = C.c_void_p(4096 + odd)
    lib, shape = K.lib(), K.ScanShape(tokens=512, channels=8, sequences=2)
    big = C.c_uint64(1 << 40)
    for f in ("bf16", "f32"):
        for which in range(4):
            o = [None] * 4
            o[which] = Q
            h0, starts, h_last, marks = o
            assert getattr(lib, "karma_k_gated_scan_fwd_" + f)(P, P, h0, starts, P, h_last, marks, C.byref(shape), P, big, None) == K.E_INVAL, (f, which)
        for which in range(5):
            o = [None, None, P, None, None]
            o[which] = Q
            h0, starts, marks, dh_last, dh0 = o
            assert getattr(lib, "karma_k_gated_scan_bwd_" + f)(P, P, h0, starts, marks, P, dh_last, P, P, dh0, C.byref(shape), P, big, None) == K.E_INVAL, (f, which)
        for name in ("tokens", "logprob", "entropy", "stats", "top_lp", "top_id"):
            assert logprob_fwd(**{**dict(fn=f, top=2, entropy=P, stats=P, top_lp=P, top_id=P), name: Q}) == K.E_INVAL, (f, name)
        for name in ("tokens", "stats", "entropy", "dl", "de"):
            assert logprob_bwd(**{**dict(fn=f), name: Q}) == K.E_INVAL, (f, name)
    ptrs = (C.c_void_p * 1)(4096 + odd)
    good = (C.c_void_p * 1)(4096)
    t = (K.AdamwTensor * 1)(K.AdamwTensor(w=4096, m=4096, v=4096, m_scale=4096, v_scale=4096, grad=4096, n=10, flags=4))
    assert lib.karma_k_adamw_states(t, 1, ptrs, good, None) == K.E_INVAL and lib.karma_k_adamw_states(t, 1, good, ptrs, None) == K.E_INVAL


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    """The operators' structures, field by field, as a C compiler lays them out."""
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    structures = dict(karma_scan_shape=K.ScanShape, karma_adamw_tensor=K.AdamwTensor, karma_adamw_step=K.AdamwStep, karma_adamw_live=K.AdamwLive)
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "karma.h"', "int main(void) {"]
    for name, s in structures.items():
        lines.append('printf("%%zu", sizeof(%s));' % name)
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (name, f[0]) for f in s._fields_] + ['printf("\\n");']
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0;", "}"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([cc, "-I", os.path.join(root, "include"), "-o", str(tmp_path / "l"), str(tmp_path / "l.c")], check=True)
    out = subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.split("\n")
    for line, (name, s) in zip(out, structures.items()):
        assert [int(v) for v in line.split()] == [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_], name


def test_a_workspace_that_is_too_small_is_refused():
    lib = K.lib()
    shape = K.ScanShape(tokens=4096, channels=64, sequences=1)
    need = K.gated_scan_ws_bytes(shape)
    assert need > 0
    for f in ("bf16", "f32"):
        for ws, size in ((P, need - 1), (P, 0), (None, need), (None, 1 << 40)):
            assert getattr(lib, "karma_k_gated_scan_fwd_" + f)(P, P, None, None, P, None, None, C.byref(shape), ws, C.c_uint64(size), None) == K.E_OOM
            assert getattr(lib, "karma_k_gated_scan_bwd_" + f)(P, P, None, None, P, P, None, P, P, None, C.byref(shape), ws, C.c_uint64(size),
                                                               None) == K.E_OOM
    need = K.token_logprob_ws_bytes(2, 100000, 20)
    assert need > 0
    for f in ("bf16", "f32"):
        for ws, size in ((P, need - 1), (P, 0), (None, need), (None, 1 << 40)):
            assert logprob_fwd(rows=2, cols=100000, top=20, top_lp=P, top_id=P, fn=f, ws=ws, ws_bytes=size) == K.E_OOM
