"""Norms of queries and keys with the rotation by position against the plain form in 64 bits: types, cuts of a head's columns, strides, places,
lengths from one token on, in place, on another stream and in a graph."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import decoder_forms as D
import paper_2008_11421_amd as K

U = D.U
EPS = 1e-5


def half(t):
    import torch
    return torch.finfo(t).eps / 2


def freqs(rot):
    return 10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))


class Case:
    """Buffers with room around them, filled with a mark that has to stay."""

    def __init__(self, t, tokens, hq, hk, hv, d, rot, pairs=False, norm=True, gap=0, off=0, positions=None, seq=0, gamma=True, seed=0, std=1.0):
        import torch
        self.t, self.tokens, self.heads, self.d, self.rot, self.pairs, self.norm = t, tokens, (hq, hk, hv), d, rot, pairs, norm
        rng = np.random.default_rng(seed)
        self.cols, self.off = sum(self.heads) * d, off
        self.ld = self.cols + gap
        self.freq = torch.from_numpy(freqs(rot)).cuda() if rot else None
        self.positions = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
        self.seq = seq
        at = np.arange(tokens) % (seq or max(tokens, 1)) if positions is None else np.asarray(positions, np.int64)
        self.angle = at[:, None].astype(np.float64) * freqs(rot)
        self.x, self.dy = self.buffer(rng, std), self.buffer(rng, 0.3)
        self.gammas = [torch.from_numpy(1 + 0.3 * rng.standard_normal(d).astype(np.float32)).to(t).cuda() if norm and gamma else None for _ in range(2)]

    def buffer(self, rng=None, std=1.0):
        import torch
        b = torch.full((self.tokens * self.ld + self.off + 64,), 7.0, dtype=self.t, device="cuda")
        if rng is not None:
            self.inside(b).copy_(torch.from_numpy((std * rng.standard_normal((self.tokens, self.cols))).astype(np.float32)).to(self.t))
        return b

    def inside(self, b):
        return b[self.off:self.off + self.tokens * self.ld].view(self.tokens, self.ld)[:, :self.cols]

    def untouched(self, b):
        c = b.clone()
        self.inside(c).fill_(7.0)
        return bool((c == 7.0).all())

    def shape(self):
        return K.QkShape(tokens=self.tokens, seq=self.seq, heads_q=self.heads[0], heads_k=self.heads[1], heads_v=self.heads[2], d=self.d, rot=self.rot,
                         flags=(K.QK_NORM if self.norm else 0) | (K.QK_PAIRS if self.pairs else 0), eps=EPS,
                         **{"ld_" + n: self.ld for n in ("q", "k", "v", "yq", "yk", "yv", "dq", "dk", "dv")})

    def parts(self, b):
        e = b.element_size()
        at = [0, self.heads[0] * self.d, (self.heads[0] + self.heads[1]) * self.d]
        return [C.c_void_p(b.data_ptr() + (self.off + a) * e) if h else None for a, h in zip(at, self.heads)]

    def fwd(self, x, y, stream=None):
        import gpu_util as g
        fn = K.lib().karma_k_qk_rotary_fwd_bf16 if x.element_size() == 2 else K.lib().karma_k_qk_rotary_fwd_f32
        p = lambda t: None if t is None else g.ptr(t)
        return fn(*self.parts(x), *map(p, self.gammas), p(self.positions), p(self.freq), *self.parts(y), C.byref(self.shape()), stream or g.stream_ptr())

    def bwd(self, dy, x, dx, dgammas=(None, None), ws=None, stream=None):
        import gpu_util as g
        fn = K.lib().karma_k_qk_rotary_bwd_bf16 if x.element_size() == 2 else K.lib().karma_k_qk_rotary_bwd_f32
        p = lambda t: None if t is None else g.ptr(t)
        return fn(*self.parts(dy), *self.parts(x)[:2], *map(p, self.gammas), p(self.positions), p(self.freq), *self.parts(dx), *map(p, dgammas),
                  C.byref(self.shape()), p(ws), C.c_uint64(0 if ws is None else ws.numel()), stream or g.stream_ptr())

    def workspace(self):
        import torch
        return torch.full((max(16, K.qk_rotary_ws_bytes(self.shape())),), 255, dtype=torch.uint8, device="cuda")

    # ---- against the plain form
    def split(self, b):
        h = self.inside(b).double().cpu().numpy().reshape(self.tokens, -1, self.d)
        return np.split(h, np.cumsum(self.heads)[:2], 1)

    def gamma64(self, k):
        return None if self.gammas[k] is None else self.gammas[k].double().cpu().numpy()

    def check_forward(self, x, y):
        for k, (xs, ys) in enumerate(zip(self.split(x)[:2], self.split(y)[:2])):
            want, bound = D.qk_forward(xs, self.gamma64(k), self.angle, self.rot, self.pairs, EPS, self.norm)
            assert (np.abs(ys - want) <= bound + half(self.t) * (np.abs(want) + bound) + 1e-37).all(), k
        assert np.array_equal(self.split(x)[2], self.split(y)[2])

    def check_backward(self, dy, x, dx, dgammas):
        for k, (gs, xs, got) in enumerate(zip(self.split(dy)[:2], self.split(x)[:2], self.split(dx)[:2])):
            want, dg, bound, terms = D.qk_backward(gs, xs, self.gamma64(k), self.angle, self.rot, self.pairs, EPS, self.norm)
            assert (np.abs(got - want) <= bound + half(self.t) * (np.abs(want) + bound) + 1e-37).all(), k
            if dgammas[k] is not None:
                # a term is off by 12 half steps of its gradient, d / 2 + 10 of the norm; a wavefront adds up a part of a token's heads for every
                # 4096th token, 6 joins of lanes, 4 of wavefronts, and of up to 1024 rows 16 and 64 follow
                chain = max(1, self.heads[k]) * (1 + self.tokens // 4096) + 6 + 4 + 16 + 64
                assert (np.abs(dgammas[k].double().cpu().numpy() - dg) <= (chain + self.d / 2 + 24) * U * terms).all(), k
        assert np.array_equal(self.split(dy)[2], self.split(dx)[2])


def types():
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}


SHAPES = [
    # tokens, query, key and value heads, d, rot, pairs, norm, gap, off
    (1, 1, 1, 0, 2, 2, False, True, 0, 0),
    (1, 32, 8, 8, 128, 128, False, True, 0, 0),
    (64, 16, 16, 16, 64, 64, False, True, 0, 0),
    (5, 3, 1, 1, 64, 64, True, True, 16, 0),
    (130, 7, 3, 0, 72, 36, True, True, 0, 0),
    (33, 4, 4, 4, 152, 152, False, True, 0, 0),
    (17, 5, 2, 0, 256, 256, False, True, 8, 8),
    (17, 2, 3, 1, 256, 128, True, True, 0, 0),
    (9, 3, 3, 0, 254, 2, False, True, 0, 0),
    (9, 2, 1, 2, 250, 126, True, True, 0, 0),
    (12, 2, 2, 0, 250, 250, False, False, 0, 0),
    (40, 6, 0, 0, 64, 0, False, True, 0, 0),
    (40, 0, 3, 2, 96, 32, False, True, 0, 0),
    (21, 4, 2, 0, 32, 32, False, False, 0, 0),
    (21, 4, 2, 1, 48, 16, True, False, 3, 1),
    (31, 2, 2, 1, 64, 64, False, True, 1, 1),
    (31, 2, 2, 1, 128, 64, True, True, 2, 2),
    (31, 2, 1, 1, 128, 120, False, True, 4, 4),
    (3, 70, 9, 1, 16, 8, False, True, 0, 0),
    (5000, 2, 1, 0, 16, 16, False, True, 0, 0),
    (9001, 1, 1, 1, 8, 4, True, True, 0, 0),
]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(int(v)) for v in s))
def test_against_the_plain_form(t, shape):
    import torch
    tokens, hq, hk, hv, d, rot, pairs, norm, gap, off = shape
    c = Case(types()[t], tokens, hq, hk, hv, d, rot, pairs, norm, gap, off, seed=tokens + d)
    x0, dy0 = c.x.clone(), c.dy.clone()
    y, dx = c.buffer(), c.buffer()
    dg = [torch.full((d,), 9.0, device="cuda") if norm else None for _ in range(2)]
    assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, c.workspace() if norm else None) == 0
    torch.cuda.synchronize()
    assert torch.equal(c.x, x0) and torch.equal(c.dy, dy0) and c.untouched(y) and c.untouched(dx)
    c.check_forward(c.x, y)
    c.check_backward(c.dy, c.x, dx, dg)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_places(t):
    """Positions of every kind, near and far, given or counted."""
    import torch
    far = [0, 1, -1, 131071, 1000003, 2 ** 31 - 1, -2 ** 31, 77777]
    for kw in (dict(positions=far), dict(seq=3), dict(seq=1), dict(seq=100)):
        c = Case(types()[t], 8, 2, 2, 0, 64, 64, seed=3, **kw)
        # 64 bits keep 2^-53 of an angle of up to 2^31, three times over
        y = c.buffer()
        assert c.fwd(c.x, y) == 0
        torch.cuda.synchronize()
        for k in range(2):
            want, bound = D.qk_forward(c.split(c.x)[k], c.gamma64(k), c.angle, 64, False, EPS)
            bound += D.partners(want, 64, False) * 3 * 2.0 ** -53 * 2.0 ** 31
            assert (np.abs(c.split(y)[k] - want) <= bound + half(c.t) * (np.abs(want) + bound)).all(), kw


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_in_place(t):
    import torch
    c = Case(types()[t], 37, 5, 3, 2, 64, 32, gap=8, seed=5)
    y, dx = c.buffer(), c.buffer()
    ws = c.workspace()
    dg, dg2 = [[torch.zeros(64, device="cuda") for _ in range(2)] for _ in range(2)]
    assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, ws) == 0
    x2, d2, x3 = c.x.clone(), c.dy.clone(), c.x.clone()
    assert c.fwd(x2, x2) == 0
    assert c.bwd(d2, c.x, d2, dg2, ws) == 0
    torch.cuda.synchronize()
    same = lambda a, b: torch.equal(c.inside(a), c.inside(b))
    assert same(x2, y) and same(d2, dx) and all(torch.equal(a, b) for a, b in zip(dg, dg2))
    c.heads = (5, 3, 0)         # (dv over v would be another matter)
    assert c.bwd(c.dy, x3, x3, dg2, ws) == 0
    torch.cuda.synchronize()
    assert torch.equal(c.inside(x3)[:, :512], c.inside(dx)[:, :512]) and all(torch.equal(a, b) for a, b in zip(dg, dg2))


def test_without_gamma_and_with_parts_of_the_gradients():
    import torch
    c = Case(torch.float32, 19, 3, 2, 0, 40, 20, gamma=False, seed=6)
    y, dx = c.buffer(), c.buffer()
    g = torch.zeros(40, device="cuda")
    assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, (None, g), c.workspace()) == 0
    torch.cuda.synchronize()
    c.check_forward(c.x, y)
    c.check_backward(c.dy, c.x, dx, (None, g))
    d2 = c.buffer()
    assert c.bwd(c.dy, c.x, d2) == 0        # no workspace without dgamma
    torch.cuda.synchronize()
    assert torch.equal(d2, dx)


def test_no_tokens():
    import torch
    c = Case(torch.float32, 0, 3, 2, 1, 40, 20)
    dg = [torch.ones(40, device="cuda") for _ in range(2)]
    assert c.fwd(c.x, c.buffer()) == 0 and c.bwd(c.dy, c.x, c.buffer(), dg, c.workspace()) == 0
    torch.cuda.synchronize()
    assert (dg[0] == 0).all() and (dg[1] == 0).all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_rows_of_zeros_and_of_extremes(t):
    import torch
    c = Case(types()[t], 6, 2, 1, 0, 64, 32, seed=8)
    h = c.inside(c.x).view(6, 3, 64)
    h[0] = 0
    h[1] *= 1e17
    h[2] *= 1e-17
    h[3, :, 1:] = 0
    y, dx = c.buffer(), c.buffer()
    dg = [torch.zeros(64, device="cuda") for _ in range(2)]
    assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, c.workspace()) == 0
    torch.cuda.synchronize()
    c.check_forward(c.x, y)
    assert (c.inside(y)[0] == 0).all()
    c.check_backward(c.dy, c.x, dx, dg)


def test_columns_that_do_not_turn_stay_bit_for_bit():
    """Without the norm: also beside infinities and NaN, and with a negative zero."""
    import torch
    for pairs in (False, True):
        c = Case(torch.bfloat16, 4, 2, 2, 0, 64, 32, pairs, norm=False, seed=9)
        h = c.inside(c.x).view(4, 4, 64)
        h[:, :, 40] = float("inf")
        h[0, :, 41] = float("nan")
        h[:, :, 42] = -0.0
        y, dx = c.buffer(), c.buffer()
        assert c.fwd(c.x, y) == 0 and c.bwd(c.x, c.x, dx) == 0
        torch.cuda.synchronize()
        bits = lambda b: c.inside(b).view(4, 4, 64)[..., 32:].contiguous().view(torch.int16)
        assert torch.equal(bits(y), bits(c.x)) and torch.equal(bits(dx), bits(c.x))
        assert torch.isfinite(c.inside(y).view(4, 4, 64)[..., :32]).all()


def test_a_bad_head_spoils_no_other():
    import torch
    c = Case(torch.float32, 3, 4, 2, 0, 64, 64, seed=10)
    y0, y1, d0, d1 = (c.buffer() for _ in range(4))
    assert c.fwd(c.x, y0) == 0 and c.bwd(c.dy, c.x, d0) == 0
    bad = c.x.clone()
    c.inside(bad).view(3, 6, 64)[1, 2, 5] = float("nan")
    assert c.fwd(bad, y1) == 0 and c.bwd(c.dy, bad, d1) == 0
    torch.cuda.synchronize()
    for a, b in ((y0, y1), (d0, d1)):
        a, b = (c.inside(t).reshape(18, 64) for t in (a, b))
        keep = torch.arange(18, device="cuda") != 8
        assert torch.equal(a[keep], b[keep]) and torch.isnan(b[8]).all()


def test_on_another_stream_and_in_two_graphs():
    import torch
    c = Case(torch.bfloat16, 300, 8, 2, 2, 128, 128, seed=11)
    y0, dx0 = c.buffer(), c.buffer()
    dg0 = [torch.zeros(128, device="cuda") for _ in range(2)]
    assert c.fwd(c.x, y0) == 0 and c.bwd(c.dy, c.x, dx0, dg0, c.workspace()) == 0
    torch.cuda.synchronize()
    sets = [(c.buffer(), c.buffer(), [torch.zeros(128, device="cuda") for _ in range(2)], c.workspace()) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, dx, dg, ws = sets[0]
        assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, ws) == 0
    side.synchronize()
    equal = lambda s: torch.equal(s[0], y0) and torch.equal(s[1], dx0) and all(torch.equal(a, b) for a, b in zip(s[2], dg0))
    assert equal(sets[0])
    graphs = []
    for y, dx, dg, ws in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, ws) == 0
        graphs.append(gr)
    for _ in range(3):
        for s in sets:
            for b in (s[0], s[1], *s[2]):
                b.fill_(7.0)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(equal(s) for s in sets)


def test_offsets_beyond_32_bits():
    import torch
    tokens, d = 3, 64
    ld = (1 << 31) + 8
    rng = np.random.default_rng(21)
    freq = torch.from_numpy(freqs(d)).cuda()
    room = lambda: torch.empty(2 * ld + d + 64, dtype=torch.bfloat16, device="cuda").as_strided((tokens, d), (ld, 1))
    x, y, dy, dx = (room() for _ in range(4))
    for t in (x, dy):
        t.copy_(torch.from_numpy(rng.standard_normal((tokens, d)).astype(np.float32)).to(torch.bfloat16))
    import gpu_util as g
    shape = K.QkShape(tokens=tokens, heads_q=1, d=d, rot=d, flags=K.QK_NORM, eps=EPS, ld_q=ld, ld_yq=ld, ld_dq=ld)
    lib = K.lib()
    assert lib.karma_k_qk_rotary_fwd_bf16(g.ptr(x), None, None, None, None, None, g.ptr(freq), g.ptr(y), None, None, C.byref(shape), g.stream_ptr()) == 0
    assert lib.karma_k_qk_rotary_bwd_bf16(g.ptr(dy), None, None, g.ptr(x), None, None, None, None, g.ptr(freq), g.ptr(dx), None, None, None, None,
                                          C.byref(shape), None, C.c_uint64(0), g.stream_ptr()) == 0
    torch.cuda.synchronize()
    angle = np.arange(tokens)[:, None] * freqs(d)
    h = lambda t: t.double().cpu().numpy().reshape(tokens, 1, d)
    want, bound = D.qk_forward(h(x), None, angle, d, False, EPS)
    assert (np.abs(h(y) - want) <= bound + half(torch.bfloat16) * (np.abs(want) + bound)).all()
    want, _, bound, _ = D.qk_backward(h(dy), h(x), None, angle, d, False, EPS)
    assert (np.abs(h(dx) - want) <= bound + half(torch.bfloat16) * (np.abs(want) + bound)).all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_gamma_of_no_heads_is_not_read(t):
    """Also where it lies on its elements' boundaries alone, while all else allows wide accesses."""
    import torch
    for heads in ((3, 0), (0, 3)):
        c = Case(types()[t], 70, *heads, 0, 128, 64, seed=22)
        other = 0 if heads[0] == 0 else 1
        outs = []
        for gamma in (None, torch.full((136,), float("nan"), dtype=c.t, device="cuda")[1:129]):
            c.gammas[other] = gamma
            y, dx, dg = c.buffer(), c.buffer(), [torch.full((128,), 9.0, device="cuda") for _ in range(2)]
            assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, c.workspace()) == 0
            torch.cuda.synchronize()
            outs.append((y, dx, *dg))
        assert all(torch.equal(a, b) for a, b in zip(*outs)) and (outs[0][2 + other] == 0).all()
        c.gammas[other] = None
        c.check_forward(c.x, outs[1][0])
        c.check_backward(c.dy, c.x, outs[1][1], outs[1][2:])


# Many tokens of many heads: a wavefront has all of a token's heads, or every second group of them, and goes around several times.
LONG = [
    # tokens, query, key and value heads, d, rot, pairs, norm, gap, off
    (8195, 9, 5, 3, 64, 32, False, True, 0, 0),
    (8195, 9, 5, 3, 152, 152, False, True, 0, 0),
    (8195, 9, 5, 3, 256, 128, True, True, 0, 0),
    (8195, 37, 5, 0, 64, 64, False, False, 0, 0),
    (8195, 9, 5, 0, 96, 0, False, True, 4, 4),
    (5501, 9, 5, 3, 128, 64, False, True, 1, 1),
    (5501, 9, 5, 0, 250, 126, True, True, 0, 0),
]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("shape", LONG, ids=lambda s: "x".join(str(int(v)) for v in s))
def test_many_tokens_of_many_heads(t, shape):
    import torch
    tokens, hq, hk, hv, d, rot, pairs, norm, gap, off = shape
    c = Case(types()[t], tokens, hq, hk, hv, d, rot, pairs, norm, gap, off, seq=777, seed=tokens + d)
    x0, dy0 = c.x.clone(), c.dy.clone()
    y, dx = c.buffer(), c.buffer()
    dg, dg2, dg3 = ([torch.full((d,), 9.0, device="cuda") if norm else None for _ in range(2)] for _ in range(3))
    ws = c.workspace() if norm else None
    assert c.fwd(c.x, y) == 0 and c.bwd(c.dy, c.x, dx, dg, ws) == 0
    torch.cuda.synchronize()
    assert torch.equal(c.x, x0) and torch.equal(c.dy, dy0) and c.untouched(y) and c.untouched(dx)
    c.check_forward(c.x, y)
    c.check_backward(c.dy, c.x, dx, dg)
    # in place: y over x, dx over dy, dx over x
    x2, d2, x3 = c.x.clone(), c.dy.clone(), c.x.clone()
    assert c.fwd(x2, x2) == 0 and c.bwd(d2, c.x, d2, dg2, ws) == 0
    same = lambda a, b: torch.equal(c.inside(a), c.inside(b))
    assert same(x2, y) and same(d2, dx) and c.untouched(x2) and c.untouched(d2)
    c.heads = (hq, hk, 0)       # (dv over v would be another matter)
    assert c.bwd(c.dy, x3, x3, dg3, ws) == 0
    torch.cuda.synchronize()
    n = (hq + hk) * d
    assert torch.equal(c.inside(x3)[:, :n], c.inside(dx)[:, :n]) and torch.equal(c.inside(x3)[:, n:], c.inside(x0)[:, n:])
    assert all(torch.equal(a, b) and torch.equal(a, e) for a, b, e in zip(dg, dg2, dg3) if norm)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_sums_for_gamma_of_large_terms_that_cancel(t):
    """With r = 1 and no rotation the terms are whole numbers, one for a token.  Wavefronts and workgroups are added up in 64 bits, each workgroup's sum is rounded to
    32 and the result is: half a step of all the terms together.  (A partial sum of 2^30 in 32 bits leaves nothing of any 1.)"""
    bound = U * (2.0 ** 31 + 998) + U * 998
    import torch
    for hq, hk in ((1, 1), (1, 0), (0, 1)):
        c = Case(types()[t], 1000, hq, hk, 0, 64, 0, gamma=False, seed=1)
        c.inside(c.x).fill_(1.0)
        c.inside(c.dy).fill_(1.0)
        c.inside(c.dy)[3] = 2.0 ** 30
        c.inside(c.dy)[996] = -2.0 ** 30
        shape = c.shape()
        shape.eps = 1e-12       # 1 / sqrt(1 + eps) is 1
        c.shape = lambda: shape
        dg = [torch.zeros(64, device="cuda") for _ in range(2)]
        assert c.bwd(c.dy, c.x, c.buffer(), dg, c.workspace()) == 0
        torch.cuda.synchronize()
        for got, h in zip(dg, (hq, hk)):
            assert ((got.double() - 998.0 * h).abs() <= bound * h).all(), (hq, hk)
