"""The gated linear recurrence on the GPU against its plain form in 64 bits: lengths from none to many carried spans, packed
sequences, strides, types, states, and the ways a program calls it (in place, on another stream, captured and replayed)."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import operator_forms as F
import paper_2008_11421_amd as K

BF16_HALF = 2.0 ** -8       # a rounding to bf16, relative


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


class Problem:
    """Inputs on both sides.  lead: elements of the allocation before the first row; pad: columns between rows; tail: rows behind the
    last sequence."""

    def __init__(self, torch, seed, tokens, channels, sequences=1, starts=None, bf16=True, state=True, pad=(0, 0, 0, 0, 0), lead=0, bias=2.0):
        self.torch, self.bf16, rng = torch, bf16, np.random.default_rng(seed)
        self.tokens, self.channels, self.sequences, self.starts = tokens, channels, sequences, starts
        self.t = torch.bfloat16 if bf16 else torch.float32
        self.pads = pad
        d = lambda a, k: self.dev(a, k, lead)
        self.gate, self.x = d(rng.standard_normal((tokens, channels)) + bias, 0), d(rng.standard_normal((tokens, channels)), 1)
        self.dh = d(rng.standard_normal((tokens, channels)), 2)
        s32 = lambda: torch.from_numpy(rng.standard_normal((sequences, channels)).astype(np.float32)).cuda()
        self.h0, self.dh_last = (s32(), s32()) if state else (None, None)
        self.h, self.dgate, self.dx = (d(np.full((tokens, channels), 7.0), k) for k in (2, 3, 4))
        self.h_last, self.dh0 = (torch.full((sequences, channels), 7.0, device="cuda") for _ in range(2))
        self.marks = torch.full((max(1, -(-tokens // K.SCAN_MARK)), channels), 7.0, device="cuda")
        self.starts_dev = torch.tensor(starts, dtype=torch.int32, device="cuda") if starts is not None else None
        self.shape = K.ScanShape(tokens=tokens, channels=channels, sequences=sequences, ld_gate=channels + pad[0], ld_x=channels + pad[1],
                                 ld_h=channels + pad[2], ld_dgate=channels + pad[3], ld_dx=channels + pad[4])
        n = K.gated_scan_ws_bytes(self.shape)
        self.ws = torch.full((max(n, 16),), 0x5A, dtype=torch.uint8, device="cuda")       # whatever it held before
        self.ws_bytes = n

    def dev(self, a, k, lead=0):
        """A tensor whose rows are pads[k] columns apart, its first element `lead` elements into the allocation."""
        a = np.asarray(a, np.float32)
        rows, ld = a.shape[0], a.shape[1] + self.pads[k]
        flat = self.torch.full((lead + max(1, rows) * ld,), 9.0, dtype=self.t, device="cuda")
        v = flat[lead:lead + rows * ld].view(rows, ld)[:, :a.shape[1]]
        v.copy_(self.torch.from_numpy(a))
        return v

    def forward(self, stream=None, marks=True, **other):
        o = lambda name: ptr(other.get(name, getattr(self, name)))
        fn = K.lib().karma_k_gated_scan_fwd_bf16 if self.bf16 else K.lib().karma_k_gated_scan_fwd_f32
        q = C.c_void_p((stream or self.torch.cuda.current_stream()).cuda_stream)
        st = fn(o("gate"), o("x"), ptr(self.h0), ptr(self.starts_dev), o("h"), o("h_last"), o("marks") if marks else None, C.byref(self.shape),
                o("ws"), C.c_uint64(self.ws_bytes), q)
        assert st == K.OK, st

    def backward(self, stream=None, **other):
        o = lambda name: ptr(other.get(name, getattr(self, name)))
        fn = K.lib().karma_k_gated_scan_bwd_bf16 if self.bf16 else K.lib().karma_k_gated_scan_bwd_f32
        q = C.c_void_p((stream or self.torch.cuda.current_stream()).cuda_stream)
        st = fn(o("gate"), o("x"), ptr(self.h0), ptr(self.starts_dev), o("marks"), o("dh"), ptr(self.dh_last), o("dgate"), o("dx"), o("dh0"),
                C.byref(self.shape), o("ws"), C.c_uint64(self.ws_bytes), q)
        assert st == K.OK, st

    def check(self, gate=None, x=None, dh=None, h=None, dgate=None, dx=None):
        """Every output against the plain form; rows behind the last sequence and the gaps between rows as they were."""
        h2 = lambda t: t.float().cpu().numpy().astype(np.float64)
        self.torch.cuda.synchronize()
        f, xs, d = h2(self.gate if gate is None else gate), h2(self.x if x is None else x), h2(self.dh if dh is None else dh)
        starts = F.starts_of(self.tokens, self.sequences, self.starts)
        h0, dl = (None if t is None else h2(t) for t in (self.h0, self.dh_last))
        hh, before, last = F.scan_forward(f, xs, starts, h0)
        dgg, dxx, first, _ = F.scan_backward(f, xs, starts, d, h0, dl)
        e = F.scan_bounds(f, xs, starts, h0, d, dl)
        n = starts[-1]
        half = BF16_HALF if self.bf16 else 0.0

        def near(name, got, want, bound):
            got = h2(got)
            assert np.isfinite(got).all(), name
            far = np.abs(got - want) - (bound + half * (np.abs(want) + bound) + 1e-37)
            assert (far <= 0).all(), (name, np.unravel_index(far.argmax(), far.shape), far.max())

        near("h", (self.h if h is None else h)[:n], hh[:n], e["h"][:n])
        near("dgate", (self.dgate if dgate is None else dgate)[:n], dgg[:n], e["dgate"][:n])
        near("dx", (self.dx if dx is None else dx)[:n], dxx[:n], e["dx"][:n])
        half = 0.0
        near("h_last", self.h_last, last, e["h_last"])
        near("dh0", self.dh0, first, e["dh0"])
        for k in range(K.SCAN_MARK, n, K.SCAN_MARK):
            if k not in starts:
                near("mark", self.marks[k // K.SCAN_MARK:][:1], before[k:k + 1], e["h"][k - 1:k])
        if h is None:
            for t, k in ((self.h, 2), (self.dgate, 3), (self.dx, 4)):
                assert (t[n:] == 7).all()
                if self.pads[k] and self.tokens > 1:
                    gap = self.torch.as_strided(t, (self.tokens - 1, self.pads[k]), (t.stride(0), 1), t.storage_offset() + self.channels)
                    assert (gap == 9).all()


def both(p):
    p.forward()
    p.backward()
    p.check()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("tokens,channels,sequences", [(1, 1, 1), (1, 130, 1), (2, 64, 2), (5, 3, 1), (31, 128, 1), (33, 127, 3), (64, 1000, 64),
                                                       (255, 66, 1), (256, 64, 1), (257, 65, 1), (511, 129, 1), (1026, 258, 2),
                                                       (1536, 256, 3), (4099, 70, 1), (2560, 8, 10), (900, 5, 300)])
def test_lengths_and_channels(torch, tokens, channels, sequences, bf16):
    both(Problem(torch, tokens + channels, tokens, channels, sequences, bf16=bf16))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("starts,tokens", [([0, 0], 3), ([0, 0, 0, 5], 5), ([0, 1, 2, 3, 700], 704), ([0, 300, 300, 301, 812, 812], 812),
                                           ([0, 256, 512, 1024, 1300], 1301), ([0, 255, 257, 258, 1279, 1281, 3000], 3007),
                                           ([0] + [7 * k for k in range(1, 100)] + [2000], 2000), ([0, 2047, 2047, 2048], 2049),
                                           (list(range(0, 601)), 600), ([0] * 80 + [40] * 90 + [600], 640)])
def test_packed_sequences(torch, starts, tokens, bf16):
    both(Problem(torch, len(starts), tokens, 96 if bf16 else 45, len(starts) - 1, starts, bf16=bf16))


@pytest.mark.parametrize("sequences,starts", [(1, None), (3, None), (2, [0, 0, 0])])
def test_no_tokens(torch, sequences, starts):
    p = Problem(torch, 5, 0, 40, sequences, starts)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    assert torch.equal(p.h_last, p.h0) and torch.equal(p.dh0, p.dh_last)


@pytest.mark.parametrize("pad,lead", [((1, 1, 1, 1, 1), 0), ((64, 64, 0, 2, 6), 0), ((3, 5, 8, 0, 1), 1), ((0, 0, 0, 0, 0), 1), ((8, 8, 8, 8, 8), 3)])
@pytest.mark.parametrize("bf16", [True, False])
def test_strides_and_alignment(torch, pad, lead, bf16):
    both(Problem(torch, 9, 700, 130, 2, pad=pad, lead=lead, bf16=bf16))


def test_without_states(torch):
    p = Problem(torch, 11, 1500, 72, 3, state=False)
    both(p)
    want = p.h.clone()
    # h_last, dh0 and marks are not wanted: the rest is the same
    p.h.fill_(7)
    p.forward(marks=False, h_last=None)
    torch.cuda.synchronize()
    assert torch.equal(p.h, want)
    dx = p.dx.clone()
    p.backward(dh0=None)
    torch.cuda.synchronize()
    assert torch.equal(p.dx, dx)


@pytest.mark.parametrize("bias", [-30.0, 8.0, 20.0])
def test_gates_that_take_or_keep(torch, bias):
    """Gates that let every input through, that keep states for thousands of tokens, and for millions."""
    both(Problem(torch, 13, 3000, 64, bias=bias, bf16=False))


def test_infinite_gates(torch):
    p = Problem(torch, 14, 600, 64, bf16=False)
    p.gate[100:110] = float("inf")
    p.gate[200:210] = float("-inf")
    both(p)
    assert torch.equal(p.h[100:110], p.h[99:100].expand(10, 64))


@pytest.mark.parametrize("tokens,sequences", [(3000, 3), (600, 6), (96, 32)])
def test_a_sequence_that_is_lost_stays_alone(torch, tokens, sequences):
    """NaN and infinities in one sequence, and in its states, reach no other."""
    p = Problem(torch, 15, tokens, 64, sequences, bf16=False)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    want = [t.clone() for t in (p.h, p.dgate, p.dx, p.h_last, p.dh0)]
    n = tokens // sequences
    p.x[n + 1] = float("nan")
    p.h0[1] = float("inf")
    p.dh_last[1] = float("nan")
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    for t, w, per in zip((p.h, p.dgate, p.dx, p.h_last, p.dh0), want, (n, n, n, 1, 1)):
        other = torch.ones(len(t), dtype=torch.bool, device="cuda")
        other[per:2 * per] = False
        assert torch.equal(t[other], w[other])
        assert not torch.isfinite(t[per:2 * per]).all()


@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("starts,tokens", [([0, 300, 1000], 1500), ([0, 1, 600], 602), ([0, 512], 1100), ([0, 4, 7], 300), ([0, 2, 2], 9)])
def test_what_lies_behind_the_last_sequence_is_not_looked_at(torch, starts, tokens, state):
    p = Problem(torch, 25, tokens, 64, len(starts) - 1, starts, state=state)
    for t, v in ((p.gate, "nan"), (p.x, "inf"), (p.dh, "nan")):
        t[starts[-1]:] = float(v)
    p.forward()
    p.backward()
    for t in (p.gate, p.x, p.dh):
        t[starts[-1]:] = 0      # (the plain form has to be able to subtract)
    p.check()


@pytest.mark.parametrize("tokens,sequences,starts", [(2100, 3, None), (64, 64, None), (2000, 4, [0, 900, 901, 901, 1990])])
def test_in_place(torch, tokens, sequences, starts):
    a = Problem(torch, 16, tokens, 132, sequences, starts)
    both(a)
    b = Problem(torch, 16, tokens, 132, sequences, starts)
    gate, x, dh, state = b.gate.clone(), b.x.clone(), b.dh.clone(), b.h0.clone()
    b.forward(h=b.x, h_last=b.h0)           # the state where it was
    torch.cuda.synchronize()
    n = (starts or [tokens])[-1]
    assert torch.equal(b.x[:n], a.h[:n]) and torch.equal(b.h0, a.h_last) and torch.equal(b.x[n:], x[n:])
    b.x.copy_(x)
    b.h0.copy_(state)
    b.forward(h=b.gate)
    torch.cuda.synchronize()
    assert torch.equal(b.gate[:n], a.h[:n])
    b.gate.copy_(gate)
    b.backward(dgate=b.gate, dx=b.dh)
    torch.cuda.synchronize()
    assert torch.equal(b.gate[:n], a.dgate[:n]) and torch.equal(b.dh[:n], a.dx[:n])
    b.gate.copy_(gate)
    b.dh.copy_(dh)
    b.backward(dgate=b.dh, dx=b.x)
    torch.cuda.synchronize()
    assert torch.equal(b.dh[:n], a.dgate[:n]) and torch.equal(b.x[:n], a.dx[:n])


@pytest.mark.parametrize("tokens,sequences", [(8192, 1), (6000, 4), (48, 48)])
def test_the_same_bits_every_time(torch, tokens, sequences):
    p = Problem(torch, 17, tokens, 520, sequences)
    both(p)
    want = [t.clone() for t in (p.h, p.dgate, p.dx, p.h_last, p.dh0, p.marks)]
    for _ in range(5):
        p.ws.random_(0, 255)
        p.forward()
        p.backward()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip((p.h, p.dgate, p.dx, p.h_last, p.dh0, p.marks), want))


def test_two_streams_at_once(torch):
    ps = [Problem(torch, 18 + k, 5000, 256, 2) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(3):
        for p, s in zip(ps, streams):
            p.forward(stream=s)
            p.backward(stream=s)
    torch.cuda.synchronize()
    for p in ps:
        p.check()


def test_captured_and_replayed(torch):
    p = Problem(torch, 20, 4000, 256, 2)
    both(p)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            p.forward(stream=side)
            p.backward(stream=side)
    rng = np.random.default_rng(21)
    for k in range(4):
        p.x.copy_(torch.from_numpy(rng.standard_normal(p.x.shape).astype(np.float32)))
        p.ws.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        p.check()


def test_tokens_one_at_a_time_are_the_sequence(torch):
    """Serving: a prompt, then single tokens with the state carried in place, against the whole sequence at once."""
    whole = Problem(torch, 22, 3 * 40, 200, 3, bf16=False)
    whole.forward()
    state = whole.h0.clone()
    view = lambda t: t.view(3, 40, 200)
    got = torch.empty_like(view(whole.h))

    def part(a, b):
        n = b - a
        gate, x = (view(t)[:, a:b].reshape(3 * n, 200).contiguous() for t in (whole.gate, whole.x))
        h = torch.empty_like(x)
        shape = K.ScanShape(tokens=3 * n, channels=200, sequences=3)
        ws = torch.empty(max(16, K.gated_scan_ws_bytes(shape)), dtype=torch.uint8, device="cuda")
        assert K.lib().karma_k_gated_scan_fwd_f32(ptr(gate), ptr(x), ptr(state), None, ptr(h), ptr(state), None, C.byref(shape), ptr(ws),
                                                  C.c_uint64(ws.numel()), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == K.OK
        got[:, a:b] = h.view(3, n, 200)

    part(0, 33)
    for t in range(33, 40):
        part(t, t + 1)
    f, x = (t.cpu().numpy() for t in (whole.gate, whole.x))
    h0 = whole.h0.cpu().numpy()
    hh, _, last = F.scan_forward(f, x, [0, 40, 80, 120], h0)
    e = F.scan_bounds(f, x, [0, 40, 80, 120], h0)
    assert (np.abs(got.view(120, 200).cpu().numpy() - hh) <= e["h"]).all()
    assert (np.abs(state.cpu().numpy() - last) <= e["h_last"]).all()


def test_a_small_workspace_is_refused(torch):
    p = Problem(torch, 23, 4096, 64)
    if p.ws_bytes:
        fn = K.lib().karma_k_gated_scan_fwd_bf16
        args = (ptr(p.gate), ptr(p.x), None, None, ptr(p.h), None, None, C.byref(p.shape))
        assert fn(*args, ptr(p.ws), C.c_uint64(p.ws_bytes - 1), None) == K.E_OOM
        assert fn(*args, None, C.c_uint64(p.ws_bytes), None) == K.E_OOM
        torch.cuda.synchronize()
        assert (p.h == 7).all()


def test_offsets_beyond_32_bits(torch):
    """A row stride that puts the last rows more than 2^32 bytes and 2^31 elements from the first."""
    tokens, channels, ld = 1500, 64, 1600000
    flat = torch.zeros(tokens * ld, dtype=torch.bfloat16, device="cuda")
    p = Problem(torch, 24, tokens, channels)
    both(p)
    wide = flat.view(tokens, ld)
    wide[:, :channels] = p.gate
    wide[:, channels:2 * channels] = p.x
    shape = K.ScanShape(tokens=tokens, channels=channels, sequences=1, ld_gate=ld, ld_x=ld, ld_h=ld)
    x, h = flat[channels:], flat[2 * channels:]
    assert K.lib().karma_k_gated_scan_fwd_bf16(ptr(flat), ptr(x), ptr(p.h0), None, ptr(h), ptr(p.h_last), None, C.byref(shape), ptr(p.ws),
                                               C.c_uint64(p.ws_bytes), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == K.OK
    torch.cuda.synchronize()
    assert torch.equal(wide[:, 2 * channels:3 * channels], p.h)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("starts,tokens,sequences,channels", [
    (None, 64 * 300, 64, 1032),                                             # whole sequences with marks at any of their tokens
    (None, 17 * 93, 17, 70), (None, 21, 1, 33), (None, 3 * 4, 3, 12), (None, 5 * 16, 5, 20),
    ([0, 250, 262, 262, 300, 513, 514, 520], 523, 7, 50),                   # packed, on both sides of a mark
    ([0] + [500 + k for k in range(40)], 539, 40, 40),                      # one long one and single tokens
    ([0] + [600 + k for k in range(40)], 639, 40, 40)])
def test_short_sequences(torch, starts, tokens, sequences, channels, bf16):
    both(Problem(torch, 26, tokens, channels, sequences, starts, bf16=bf16))


def test_nothing_where_nothing_is_needed(torch):
    """No workspace where a call needs none, and no tensors where there are no tokens."""
    p = Problem(torch, 27, 200, 40)
    assert K.gated_scan_ws_bytes(p.shape) == 0
    p.ws = None
    both(p)
    e = Problem(torch, 28, 0, 40, 3)
    e.ws = None
    e.forward(marks=False, gate=None, x=None, h=None)
    e.backward(gate=None, x=None, marks=None, dh=None, dgate=None, dx=None)
    torch.cuda.synchronize()
    assert torch.equal(e.h_last, e.h0) and torch.equal(e.dh0, e.dh_last)


def check_closely(p):
    """Every output within the bounds that hold where no bit is lost to cancellation."""
    h2 = lambda t: t.float().cpu().numpy().astype(np.float64)
    p.torch.cuda.synchronize()
    starts, n = F.starts_of(p.tokens, p.sequences, p.starts), F.starts_of(p.tokens, p.sequences, p.starts)[-1]
    h0, dl = (None if t is None else h2(t) for t in (p.h0, p.dh_last))
    want, bound = F.scan_by_shares(h2(p.gate), h2(p.x), starts, h0, h2(p.dh), dl)
    for name in want:
        rows = n if name in ("h", "dgate", "dx") else None
        got, w, e = h2(getattr(p, name))[:rows], want[name][:rows], bound[name][:rows]
        if p.bf16 and rows is not None:
            e = e + BF16_HALF * (np.abs(w) + e) + 1e-38
        far = np.abs(got - w) - e
        assert (far <= 0).all(), (name, np.unravel_index(far.argmax(), far.shape), far.max())


SHAPES = [(700, 2, None), (1600, 4, [0, 300, 300, 301, 1590]), (48, 48, None), (5, 1, None)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("bias", [-30.0, -16.0, -10.0, -3.0, 0.0, 6.0])
@pytest.mark.parametrize("tokens,sequences,starts", SHAPES)
def test_no_bits_are_lost_on_either_side_of_the_gate(torch, tokens, sequences, starts, bias, bf16):
    p = Problem(torch, 30, tokens, 68, sequences, starts, bf16=bf16, bias=bias)
    p.forward()
    p.backward()
    check_closely(p)


@pytest.mark.parametrize("tokens,sequences,starts", SHAPES)
def test_large_states_that_a_gate_lets_go_of(torch, tokens, sequences, starts):
    """States of 1e8, and inputs of 3e4 on the way, that a gate of -30, -10 or minus infinity replaces by inputs of a thousandth."""
    p = Problem(torch, 31, tokens, 68, sequences, starts, bf16=False, bias=1.0)
    rng = np.random.default_rng(32)
    p.h0.mul_(1e8)
    p.x.mul_(1e-3)
    at = torch.from_numpy(rng.integers(0, tokens, tokens // 8)).cuda()
    p.x[at] = 3e4
    for k, gate in enumerate((-30.0, -10.0, float("-inf"))):
        p.gate[k::7] = gate
    p.forward()
    p.backward()
    # (minus infinity: an exponential of nothing, the input itself)
    p.gate.clamp_(min=-200.0)
    check_closely(p)
    if tokens == 48:
        assert torch.equal(p.h[2::7], p.x[2::7])


@pytest.mark.parametrize("starts", [None, [0, 100, 357]])
@pytest.mark.parametrize("bf16", [True, False])
def test_more_blocks_of_channels_than_workgroups_that_run_at_once(torch, bf16, starts):
    """300 000 channels of some chunks: workgroups of all blocks can never be there together.  The same bits as calls on a part of the
    channels, and within bounds."""
    tokens, channels = 600, 300_032
    t = torch.bfloat16 if bf16 else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(40)
    make = lambda rows=tokens, dtype=t, mean=0.0: torch.empty((rows, channels), device="cuda", dtype=dtype).normal_(mean, 1.0, generator=gen)
    S = 1 if starts is None else len(starts) - 1
    gate, x, dh, h0, dh_last = make(mean=3.0), make(), make(), make(S, torch.float32), make(S, torch.float32)
    st = torch.tensor(starts, dtype=torch.int32, device="cuda") if starts else None
    n = starts[-1] if starts else tokens
    fwd, bwd = ((K.lib().karma_k_gated_scan_fwd_bf16, K.lib().karma_k_gated_scan_bwd_bf16) if bf16 else
                (K.lib().karma_k_gated_scan_fwd_f32, K.lib().karma_k_gated_scan_bwd_f32))
    q = C.c_void_p(torch.cuda.current_stream().cuda_stream)

    def call(first, count):
        cut = lambda a: a[:, first:first + count]
        a, b, d, s, l = cut(gate), cut(x), cut(dh), cut(h0).contiguous(), cut(dh_last).contiguous()
        out = lambda rows=tokens, dtype=t: torch.zeros((rows, count), device="cuda", dtype=dtype)
        h, dgate, dx, last, first_g, marks = out(), out(), out(), out(S, torch.float32), out(S, torch.float32), out(3, torch.float32)
        shape = K.ScanShape(tokens=tokens, channels=count, sequences=S, ld_gate=channels, ld_x=channels, ld_h=count)
        ws = torch.empty(K.gated_scan_ws_bytes(shape), dtype=torch.uint8, device="cuda")
        assert fwd(ptr(a), ptr(b), ptr(s), ptr(st), ptr(h), ptr(last), ptr(marks), C.byref(shape), ptr(ws), C.c_uint64(ws.numel()), q) == K.OK
        if count < channels:
            d = d.contiguous()
        assert bwd(ptr(a), ptr(b), ptr(s), ptr(st), ptr(marks), ptr(d), ptr(l), ptr(dgate), ptr(dx), ptr(first_g), C.byref(shape), ptr(ws),
                   C.c_uint64(ws.numel()), q) == K.OK
        torch.cuda.synchronize()
        return dict(h=h, dgate=dgate, dx=dx, h_last=last, dh0=first_g)

    whole = call(0, channels)
    for first in (0, 131_072, channels - 2048):
        part = call(first, 2048)
        for k in part:
            assert torch.equal(whole[k][:, first:first + 2048], part[k]), (k, first)
    some = torch.arange(7, channels, channels // 40, device="cuda")
    h2 = lambda a: a[:, some].float().cpu().numpy().astype(np.float64)
    want, bound = F.scan_by_shares(h2(gate), h2(x), F.starts_of(tokens, S, starts), h2(h0), h2(dh), h2(dh_last))
    for k in want:
        rows = n if k in ("h", "dgate", "dx") else None
        got, w, e = h2(whole[k])[:rows], want[k][:rows], bound[k][:rows]
        if bf16 and rows:
            e = e + BF16_HALF * (np.abs(w) + e) + 1e-38
        assert (np.abs(got - w) <= e).all(), k


@pytest.mark.parametrize("bf16,tokens,channels,sequences", [(True, 256 * 100 + 3, 260, 1), (False, 256 * 17, 130, 2), (True, 256 * 9, 64, 1), (True, 256 * 8 + 1, 64, 1),
                                                            (True, 256 * 16 + 1, 64, 1), (True, 256 * 33, 65, 3)])
def test_groups_of_chunks(torch, bf16, tokens, channels, sequences):
    """Chunks that fill their groups, end one, and begin the next."""
    p = Problem(torch, 41, tokens, channels, sequences, bf16=bf16, bias=7.0)     # states live for a thousand tokens
    p.forward()
    p.backward()
    check_closely(p)


def test_beside_work_that_fills_the_device(torch):
    p = Problem(torch, 42, 20000, 512, 1, bias=6.0)
    both(p)
    want = [t.clone() for t in (p.h, p.dgate, p.dx, p.h_last, p.dh0)]
    a = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            for _ in range(4):
                b = a @ a
        p.forward(stream=other)
        p.backward(stream=other)
    torch.cuda.synchronize()
    assert torch.isfinite(b).all()
    assert all(torch.equal(t, w) for t, w in zip((p.h, p.dgate, p.dx, p.h_last, p.dh0), want))


@pytest.mark.parametrize("tokens,sequences,starts", SHAPES)
@pytest.mark.parametrize("states", [(False, False), (True, False), (False, True), (True, True)])
def test_any_of_the_states_may_be_missing(torch, tokens, sequences, starts, states):
    """h0 and dh_last, each with and without; and neither last states nor their gradients asked for: the rest is the same, from outputs that
    held something else."""
    p = Problem(torch, 50, tokens, 70, sequences, starts, state=True)
    if not states[0]:
        p.h0 = None
    if not states[1]:
        p.dh_last = None
    both(p)
    want = [t.clone() for t in (p.h, p.dgate, p.dx)]
    for t in (p.h, p.dgate, p.dx, p.h_last, p.dh0):
        t.fill_(7)
    p.forward(h_last=None)
    p.backward(dh0=None)
    torch.cuda.synchronize()
    for t, w in zip((p.h, p.dgate, p.dx), want):
        assert torch.equal(t, w) and not (t == 7).all()
    assert (p.h_last == 7).all() and (p.dh0 == 7).all()


@pytest.mark.parametrize("bf16,each,sequences,channels", [(True, 300, 1030, 64), (False, 512, 520, 66), (True, 192, 520, 60), (False, 97, 2, 33), (True, 96, 2, 70),
                                                          (True, 128, 3, 70)])
def test_many_whole_sequences(torch, bf16, each, sequences, channels):
    """Sequences that are taken whole although marks lie inside them, and lengths next to the borders of that rule: some of the sequences
    against the plain form, forward and, from the marks, backward."""
    t = torch.bfloat16 if bf16 else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(60)
    tokens = each * sequences
    make = lambda rows, mean=0.0, dtype=t: torch.empty((rows, channels), device="cuda", dtype=dtype).normal_(mean, 1.0, generator=gen)
    p = Problem(torch, 61, 1, channels, bf16=bf16)
    p.tokens, p.sequences = tokens, sequences
    p.gate, p.x, p.dh, p.h0, p.dh_last = make(tokens, 3.0), make(tokens), make(tokens), make(sequences, dtype=torch.float32), make(sequences, dtype=torch.float32)
    p.h, p.dgate, p.dx, p.h_last, p.dh0 = (torch.zeros_like(a) for a in (p.gate, p.gate, p.gate, p.h0, p.h0))
    p.marks = torch.zeros((-(-tokens // K.SCAN_MARK), channels), device="cuda")
    p.shape = K.ScanShape(tokens=tokens, channels=channels, sequences=sequences)
    p.ws_bytes = K.gated_scan_ws_bytes(p.shape)
    p.ws = torch.full((max(16, p.ws_bytes),), 0x5A, dtype=torch.uint8, device="cuda")
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    h2 = lambda a: a.float().cpu().numpy().astype(np.float64)
    for j in {0, 1, sequences // 2, sequences - 1}:
        rows = slice(j * each, (j + 1) * each)
        want, bound = F.scan_by_shares(h2(p.gate[rows]), h2(p.x[rows]), [0, each], h2(p.h0[j:j + 1]), h2(p.dh[rows]), h2(p.dh_last[j:j + 1]))
        for k in want:
            wide = k in ("h", "dgate", "dx")
            got, e = h2(getattr(p, k)[rows] if wide else getattr(p, k)[j:j + 1]), bound[k]
            if bf16 and wide:
                e = e + BF16_HALF * (np.abs(want[k]) + e) + 1e-38
            assert (np.abs(got - want[k]) <= e).all(), (k, j)
        for r in range(-(-rows.start // K.SCAN_MARK) * K.SCAN_MARK, rows.stop, K.SCAN_MARK):
            if r > rows.start:
                at = r - rows.start - 1
                assert (np.abs(h2(p.marks[r // K.SCAN_MARK]) - want["h"][at]) <= bound["h"][at]).all(), (j, r)
