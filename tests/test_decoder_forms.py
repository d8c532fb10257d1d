"""The plain forms of the norms of queries and keys with rotation, of drawing tokens and of the global gradient norm: gradients against
central differences, closed forms, and what the entry points refuse (no GPU is needed for a refusal)."""
import ctypes as C
import math

import numpy as np
import pytest

import decoder_forms as D
import paper_2008_11421_amd as K

P = C.c_void_p(4096)        # a pointer that no call here may follow
u64 = C.c_uint64


@pytest.mark.parametrize("rot,pairs,norm", [(8, False, True), (4, True, True), (0, False, True), (8, True, False), (6, False, False)])
def test_qk_gradients_against_differences(rot, pairs, norm):
    rng = np.random.default_rng(rot + pairs)
    x, dy, gamma = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8)), rng.standard_normal(8) if norm else None
    angle = rng.standard_normal((3, rot // 2)) * 3
    loss = lambda x, gamma: (D.qk_forward(x, gamma, angle, rot, pairs, 1e-3, norm)[0] * dy).sum()
    dx, dgamma, _, _ = D.qk_backward(dy, x, gamma, angle, rot, pairs, 1e-3, norm)
    for k, (a, got) in enumerate(((x, dx), (gamma, dgamma)) if norm else ((x, dx),)):
        for i in np.ndindex(a.shape):
            args = [x.copy(), None if gamma is None else gamma.copy()]
            args[k][i] += 1e-5
            up = loss(*args)
            args[k][i] -= 2e-5
            # the differences are off by h^2 / 6 times the third derivative (a few tens at most) and 1e-15 / h
            assert abs(got[i] - (up - loss(*args)) / 2e-5) < 1e-8, (k, i)


def test_a_rotation_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    freq = 100.0 ** (-np.arange(8) / 8)
    at = lambda v, p, pairs: D.turn(v, np.array([[p]]) * freq, 16, pairs)
    for pairs in (False, True):
        assert np.allclose((at(q, 5, pairs) ** 2).sum(), (q ** 2).sum())
        assert np.allclose((at(q, 7, pairs) * at(k, 3, pairs)).sum(), (at(q, 1004, pairs) * at(k, 1000, pairs)).sum())


def test_sample_closed_forms():
    z = np.zeros(8)
    for j in range(8):
        assert D.sample_row(z, 1.0, 1.0, 0.0, 0, j / 8) == (j, -math.log(8), 8)
    assert D.sample_row(z, 1.0, 0.5, 0.0, 0, 0.99)[::2] == (3, 4)           # the first half by index
    assert D.sample_row(z, 1.0, 0.51, 0.0, 0, 0.99)[::2] == (4, 5)
    assert D.sample_row(z, 1.0, 0.5, 0.0, 3, 0.99)[::2] == (1, 2)           # half of the first three
    z = np.log(np.array([1.0, 4.0, 2.0, 1.0]))
    assert D.sample_row(z, 1.0, 1.0, 0.3, 0, 0.0)[::2] == (1, 2)
    assert D.sample_row(z, 1.0, 1.0, 0.3, 0, 0.7)[::2] == (2, 2)
    assert D.sample_row(z, 0.0, 1.0, 0.0, 0, 0.7) == (1, 0.0, 1)
    assert D.sample_row(z, 1.0, 0.0, 0.0, 0, 0.7)[::2] == (1, 1)
    assert D.sample_row(np.full(3, -np.inf), 1.0, 1.0, 0.0, 0, 0.5)[0] == -1


def test_grad_norm_closed_forms():
    norm, factor, each = D.grad_norm([[3.0], [4.0]], 1.0, 1.0)
    assert norm == 5 and factor == 1 / 5 and each == [3, 4]
    assert D.grad_norm([[3.0], []], 10.0, 0.5)[:2] == (1.5, 0.5)
    assert D.grad_norm([[math.inf]], 10.0, 1.0)[1] == 0 and math.isnan(D.grad_norm([[math.nan]], 10.0, 1.0)[1])


# ------------------------------------------------------------------------------------------------- refusals
GOOD = dict(tokens=4, heads_q=2, heads_k=2, heads_v=0, d=64, rot=64, flags=K.QK_NORM, eps=1e-6)
FWD = dict(q=P, k=P, v=None, gamma_q=P, gamma_k=P, positions=None, freq=P, yq=P, yk=P, yv=None)
BWD = dict(dyq=P, dyk=P, dyv=None, q=P, k=P, gamma_q=P, gamma_k=P, positions=None, freq=P, dq=P, dk=P, dv=None, dgq=P, dgk=P)


def qk_fwd(fn="bf16", shape=None, **change):
    s = K.QkShape(**{**GOOD, **(shape or {})})
    return getattr(K.lib(), "karma_k_qk_rotary_fwd_" + fn)(*{**FWD, **change}.values(), C.byref(s), None)


def qk_bwd(fn="bf16", shape=None, ws=P, ws_bytes=1 << 40, **change):
    s = K.QkShape(**{**GOOD, **(shape or {})})
    return getattr(K.lib(), "karma_k_qk_rotary_bwd_" + fn)(*{**BWD, **change}.values(), C.byref(s), ws, u64(ws_bytes), None)


def test_qk_refusals():
    assert K.lib().karma_k_qk_rotary_fwd_bf16(*FWD.values(), None, None) == K.E_INVAL
    assert K.lib().karma_k_qk_rotary_bwd_f32(*BWD.values(), None, P, u64(1 << 40), None) == K.E_INVAL
    for bad in (dict(d=0), dict(d=63), dict(d=258), dict(rot=66), dict(rot=31), dict(rot=0, flags=0), dict(flags=4 | K.QK_NORM), dict(heads_q=0, heads_k=0),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(ld_q=127), dict(ld_yk=64), dict(ld_dq=1), dict(ld_k=1 << 62),
                dict(tokens=1 << 26), dict(seq=1 << 26), dict(heads_q=(1 << 14) + 1), dict(heads_v=(1 << 14) + 1), dict(heads_v=1, ld_v=63),
                dict(heads_v=1, ld_dv=63)):
        assert qk_fwd(shape=bad) == K.E_INVAL and qk_bwd(shape=bad) == K.E_INVAL, bad
        assert K.qk_rotary_ws_bytes(K.QkShape(**{**GOOD, **bad})) == 0, bad
    for f, odd in (("bf16", 1), ("f32", 2)):
        Q = C.c_void_p(4096 + odd)
        for name in ("q", "k", "freq", "yq", "yk"):
            assert qk_fwd(f, **{name: None}) == K.E_INVAL, name
        for name in ("q", "k", "freq", "yq", "yk", "gamma_q", "gamma_k", "positions"):
            assert qk_fwd(f, **{name: Q}) == K.E_INVAL, name
        for name in ("q", "k", "freq", "dyq", "dyk", "dq", "dk"):
            assert qk_bwd(f, **{name: None}) == K.E_INVAL, name
        for name in ("q", "k", "freq", "dyq", "dyk", "dq", "dk", "gamma_q", "gamma_k", "positions", "dgq", "dgk"):
            assert qk_bwd(f, **{name: Q}) == K.E_INVAL, name
        v = dict(heads_v=2)
        assert qk_fwd(f, v) == K.E_INVAL and qk_fwd(f, v, v=P) == K.E_INVAL and qk_fwd(f, v, v=Q, yv=P) == K.E_INVAL
        assert qk_bwd(f, v) == K.E_INVAL and qk_bwd(f, v, dyv=P) == K.E_INVAL and qk_bwd(f, v, dyv=P, dv=Q) == K.E_INVAL
    # gamma and its gradient belong to the norm
    plain = dict(flags=0)
    assert qk_fwd(shape=plain) == K.E_INVAL and qk_bwd(shape=plain, gamma_q=None, gamma_k=None) == K.E_INVAL
    # in place with other strides than the input's
    assert qk_fwd(shape=dict(ld_q=256), yq=P) == K.E_INVAL
    other = C.c_void_p(8192)
    assert qk_bwd(shape=dict(ld_yq=256), dq=P, q=other) == K.E_INVAL and qk_bwd(shape=dict(ld_q=256), dyq=other) == K.E_INVAL
    need = K.qk_rotary_ws_bytes(K.QkShape(**GOOD))
    assert need > 0
    for f in ("bf16", "f32"):
        for ws, size in ((P, need - 1), (P, 0), (None, need), (None, 1 << 40)):
            assert qk_bwd(f, ws=ws, ws_bytes=size) == K.E_OOM
        assert qk_bwd(f, ws=C.c_void_p(4104)) == K.E_INVAL
    none = dict(tokens=0)
    assert qk_fwd(shape=none, q=None, k=None, yq=None, yk=None, freq=None) == K.OK
    assert qk_bwd(shape=none, dyq=None, dyk=None, q=None, k=None, dq=None, dk=None, freq=None, dgq=None, dgk=None, ws=None) == K.OK


def sample(rows=4, cols=100, ld=0, rules=P, n_rules=1, logits=P, uniform=P, token=P, logprob=P, kept=P, fn="bf16", ws=None, ws_bytes=0):
    return getattr(K.lib(), "karma_k_sample_" + fn)(logits, u64(ld), rules, C.c_uint32(n_rules), uniform, token, logprob, kept, C.c_uint32(rows),
                                                    C.c_uint32(cols), ws, u64(ws_bytes), None)


def test_sample_refusals():
    for bad in (dict(cols=0), dict(cols=K.SAMPLE_COLS_MAX + 1), dict(ld=99), dict(ld=1 << 62), dict(rows=1 << 20), dict(n_rules=0), dict(n_rules=3), dict(rules=None),
                dict(uniform=None), dict(logits=None), dict(token=None, logprob=None, kept=None), dict(logits=C.c_void_p(4097)),
                dict(logits=C.c_void_p(4098), fn="f32")):
        assert sample(**bad) == K.E_INVAL, bad
    for name in ("rules", "uniform", "token", "logprob", "kept"):
        for odd in (1, 2, 3):
            for f in ("bf16", "f32"):
                assert sample(**{"fn": f, name: C.c_void_p(4096 + odd)}) == K.E_INVAL, (name, odd)
    assert sample(rows=0, n_rules=0, logits=None, rules=None, uniform=None) == K.OK


def test_grad_refusals():
    lib = K.lib()
    good = dict(grad=4096, out=8192, n=10, flags=0)
    call = lambda max_norm=1.0, scale=1.0, norm=P, each=P, factor=P, ws=P, ws_bytes=1 << 40, n=1, **change: lib.karma_k_grad_norm(
        (K.GradTensor * 1)(K.GradTensor(**{**good, **change})) if n else None, n, C.c_float(max_norm), C.c_float(scale), norm, each, factor, ws,
        u64(ws_bytes), None)
    clip = lambda factor=P, **change: lib.karma_k_grad_clip((K.GradTensor * 1)(K.GradTensor(**{**good, **change})), 1, factor, None)
    assert lib.karma_k_grad_norm(None, 1, C.c_float(1), C.c_float(1), P, P, P, P, u64(1 << 40), None) == K.E_INVAL
    assert lib.karma_k_grad_clip(None, 1, P, None) == K.E_INVAL and lib.karma_k_grad_clip(None, 0, P, None) == K.OK
    for bad in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(norm=None, each=None, factor=None), dict(norm=C.c_void_p(4098)), dict(each=C.c_void_p(4097)),
                dict(factor=C.c_void_p(4098)), dict(grad=None), dict(grad=4098), dict(grad=4097, flags=1), dict(flags=4), dict(n=1 << 36), dict(ws=C.c_void_p(4104))):
        if "n" in bad:
            t = (K.GradTensor * 1)(K.GradTensor(**{**good, **bad}))
            assert lib.karma_k_grad_norm(t, 1, C.c_float(1), C.c_float(1), P, P, P, P, u64(1 << 60), None) == K.E_INVAL
            assert K.grad_norm_ws_bytes(t) == 0 and lib.karma_k_grad_clip(t, 1, P, None) == K.E_INVAL
        else:
            assert call(**bad) == K.E_INVAL, bad
    t = (K.GradTensor * 2)(K.GradTensor(**{**good, "n": 1 << 35}), K.GradTensor(**good))        # too many together
    assert K.grad_norm_ws_bytes(t) == 0 and lib.karma_k_grad_clip(t, 2, P, None) == K.E_INVAL
    need = K.grad_norm_ws_bytes((K.GradTensor * 1)(K.GradTensor(**good)))
    assert need > 0
    for ws, size in ((P, need - 1), (None, 1 << 40), (P, 0)):
        assert call(ws=ws, ws_bytes=size) == K.E_OOM
    for bad in (dict(factor=None), dict(factor=C.c_void_p(4098)), dict(out=None), dict(out=8194), dict(out=8193, flags=2), dict(grad=None), dict(grad=4097, flags=1)):
        assert clip(**bad) == K.E_INVAL, bad
    assert clip(n=0, grad=None, out=None) == K.OK


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    structures = dict(karma_qk_shape=K.QkShape, karma_sample_rule=K.SampleRule, karma_grad_tensor=K.GradTensor)
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


def test_a_norm_that_launches_nothing_reports_no_error_of_others():
    """No tensors and only norms of each wanted: there is nothing to do, whatever became of the calls before."""
    assert K.lib().karma_k_grad_norm(None, 0, C.c_float(1), C.c_float(1), None, P, None, P, u64(8), None) == K.OK


def test_clipping_in_place_needs_one_type():
    """A gradient that becomes a value of another size at the same place would be written over before it is read."""
    one = lambda flags, **change: K.lib().karma_k_grad_clip((K.GradTensor * 2)(K.GradTensor(grad=8192, out=12288, n=4, flags=0),
                                                                                 K.GradTensor(**{**dict(grad=4096, out=4096, n=10, flags=flags), **change})), 2, P, None)
    assert one(K.GRAD_OUT_BF16) == K.E_INVAL and one(K.GRAD_BF16) == K.E_INVAL
    # (the norm does not look at the outputs, nor clipping at those of no values)
    empty = (K.GradTensor * 1)(K.GradTensor(grad=4096, out=4096, n=0, flags=K.GRAD_OUT_BF16))
    assert K.lib().karma_k_grad_clip(empty, 1, P, None) == K.OK
    assert K.grad_norm_ws_bytes((K.GradTensor * 1)(K.GradTensor(grad=4096, out=4096, n=10, flags=K.GRAD_OUT_BF16))) > 0
