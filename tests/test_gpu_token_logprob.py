"""Log probabilities, entropies, alternatives and their gradient on the GPU against the plain form in 64 bits."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import operator_forms as F
import paper_2008_11421_amd as K

NEG = float("-inf")


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


class Problem:
    def __init__(self, torch, seed, rows, cols, bf16=True, top=0, scale=1.0, pad=0, pad_d=0, lead=0, spread=3.0, z=None):
        self.torch, self.rows, self.cols, self.bf16, self.top, self.scale = torch, rows, cols, bf16, top, float(np.float32(scale))
        rng = np.random.default_rng(seed)
        self.t = torch.bfloat16 if bf16 else torch.float32
        z = rng.standard_normal((rows, cols)) * spread if z is None else z
        self.flat = torch.full((lead + rows * (cols + pad),), 9.0, dtype=self.t, device="cuda")
        self.z = self.flat[lead:].view(rows, cols + pad)[:, :cols]
        self.z.copy_(torch.from_numpy(np.asarray(z, np.float32)))
        tokens = rng.integers(0, cols, rows)
        tokens[1::5] = -1
        tokens[3::7] = cols          # one past the last: no column either
        self.tokens = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        f = lambda *s: torch.full(s, 7.0, device="cuda")
        self.logprob, self.entropy, self.stats, self.top_logprob = f(rows), f(rows), f(rows, 2), f(rows, top)
        self.top_id = torch.full((rows, top), 7, dtype=torch.int32, device="cuda")
        self.dlogprob, self.dentropy = (torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda() for _ in range(2))
        self.dflat = torch.full((lead + rows * (cols + pad_d),), 9.0, dtype=self.t, device="cuda")
        self.d = self.dflat[lead:].view(rows, cols + pad_d)[:, :cols]
        self.ws_bytes = K.token_logprob_ws_bytes(rows, cols, top)
        self.ws = torch.full((max(16, self.ws_bytes),), 0x5A, dtype=torch.uint8, device="cuda")

    def q(self, stream):
        return C.c_void_p((stream or self.torch.cuda.current_stream()).cuda_stream)

    def forward(self, stream=None, **other):
        o = lambda name: ptr(other.get(name, getattr(self, name)))
        fn = K.lib().karma_k_token_logprob_fwd_bf16 if self.bf16 else K.lib().karma_k_token_logprob_fwd_f32
        st = fn(ptr(self.z), C.c_uint64(self.z.stride(0)), o("tokens"), o("logprob"), o("entropy"), o("stats"), o("top_logprob") if self.top else None,
                o("top_id") if self.top else None, self.rows, self.cols, self.top, C.c_float(self.scale), o("ws"), C.c_uint64(self.ws_bytes), self.q(stream))
        assert st == K.OK, st

    def backward(self, stream=None, **other):
        o = lambda name: ptr(other.get(name, getattr(self, name)))
        fn = K.lib().karma_k_token_logprob_bwd_bf16 if self.bf16 else K.lib().karma_k_token_logprob_bwd_f32
        d = other.get("d", self.d)
        st = fn(ptr(self.z), C.c_uint64(self.z.stride(0)), o("tokens"), o("stats"), o("entropy"), o("dlogprob"), o("dentropy"), ptr(d),
                C.c_uint64(d.stride(0)), self.rows, self.cols, C.c_float(self.scale), self.q(stream))
        assert st == K.OK, st

    def check_forward(self):
        self.torch.cuda.synchronize()
        z, tokens = self.z.float().cpu().numpy().astype(np.float64), self.tokens.cpu().numpy()
        e, r = F.logprob_bounds(z, self.scale), F.logprob_forward(z, tokens, self.scale, self.top)
        live = ~r["empty"]
        named = (tokens >= 0) & (tokens < self.cols)
        at = np.where(named, tokens, 0)

        def near(name, got, want, bound):
            got = got.cpu().numpy().astype(np.float64)
            same = got == want
            with np.errstate(invalid="ignore"):
                assert (same | (np.abs(got - want) <= bound)).all(), (name, got, want, bound)

        near("logprob", self.logprob, r["logprob"], np.where(named, e["q"][np.arange(self.rows), at], 0))
        near("entropy", self.entropy, r["entropy"], np.where(live, e["entropy"], 0))
        assert np.array_equal(self.stats[:, 0].cpu().numpy(), r["stats"][:, 0].astype(np.float32))
        near("ln s", self.stats[:, 1], r["stats"][:, 1], np.where(live, e["ls"], 0))
        if self.top:
            assert np.array_equal(self.top_id.cpu().numpy(), r["top_id"])
            near("top", self.top_logprob, r["top_logprob"], np.take_along_axis(e["q"], r["top_id"], 1))

    def check_backward(self, d=None, dlogprob=True, dentropy=True, z=None):
        self.torch.cuda.synchronize()
        z, tokens = (self.z if z is None else z).float().cpu().numpy().astype(np.float64), self.tokens.cpu().numpy()
        dl, de = (t.cpu().numpy().astype(np.float64) if on else None for t, on in ((self.dlogprob, dlogprob), (self.dentropy, dentropy)))
        want = F.logprob_backward(z, tokens, self.scale, dl, de)
        e = F.logprob_bounds(z, self.scale)
        p, q, H = e["p"], np.where(e["p"] > 0, e["forward"]["q"], 0.0), e["forward"]["entropy"][:, None]
        # p is off by its exponential and its argument, and below the smallest normal number of fp32 (2^-126) it may be 0: an exponential
        # of less has no more bits to give; each product and sum by a rounding
        ep = p * (e["q"] + 8 * F.U) + np.where(p < 2.0 ** -125, 2.0 ** -126, 0.0)
        bound = np.zeros_like(p)
        if dl is not None:
            bound += np.abs(dl)[:, None] * (ep + 2 * F.U * p)
        if de is not None:
            bound += np.abs(de)[:, None] * (ep * np.abs(q + H) + p * (e["q"] + e["entropy"][:, None]) + 4 * F.U * p * (np.abs(q) + np.abs(H)))
        bound = self.scale * bound + 4 * F.U * np.abs(want) + 4 * F.U * self.scale * (0 if dl is None else np.abs(dl)[:, None] * (p + 1e-30))
        bound = bound + (2.0 ** -8 if self.bf16 else 0) * (np.abs(want) + bound) + 1e-37
        got = (self.d if d is None else d).float().cpu().numpy().astype(np.float64)
        assert np.isfinite(got).all()
        # a token's own element is a difference of dlogprob and its share of it
        hit = np.zeros_like(p, bool)
        named = (tokens >= 0) & (tokens < self.cols)
        hit[np.arange(self.rows)[named], tokens[named]] = True
        if dl is not None:
            bound = bound + hit * 2 * F.U * np.abs(dl)[:, None] * self.scale
        far = np.abs(got - want) - bound
        assert (far <= 0).all(), (np.unravel_index(far.argmax(), far.shape), far.max())

    def gaps(self):
        for flat, v in ((self.flat, self.z), (self.dflat, self.d)):
            pad = v.stride(0) - self.cols
            if pad and self.rows:
                at = v.storage_offset() + self.cols
                assert (self.torch.as_strided(flat, (self.rows, pad), (v.stride(0), 1), at) == 9).all()


def both(p):
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()
    p.gaps()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,cols,top", [(1, 1, 1), (3, 2, 2), (1, 7, 7), (5, 8, 3), (130, 9, 5), (2, 63, 63), (4, 64, 64), (7, 65, 64), (33, 255, 1),
                                           (40, 1000, 20), (600, 513, 4), (1, 4096, 50), (3, 10007, 20), (2, 51200, 20), (9, 32000, 5), (1, 160001, 64),
                                           (1100, 2050, 3), (300, 2048, 0)])
def test_rows_and_columns(torch, rows, cols, top, bf16):
    both(Problem(torch, rows + cols, rows, cols, bf16, top))


@pytest.mark.parametrize("pad,pad_d,lead", [(1, 1, 0), (8, 8, 8), (3, 0, 1), (0, 5, 3), (7, 7, 5)])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,cols", [(20, 1003), (600, 2001)])
def test_strides_and_alignment(torch, rows, cols, pad, pad_d, lead, bf16):
    both(Problem(torch, 3, rows, cols, bf16, 6, pad=pad, pad_d=pad_d, lead=lead))


@pytest.mark.parametrize("scale", [0.05, 0.7, 1.4, 25.0])
def test_temperatures(torch, scale):
    both(Problem(torch, 4, 33, 3001, False, 5, scale))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows", [8, 1200])
def test_masked_logits(torch, rows, bf16):
    """Columns that are not allowed, rows that have one or none allowed, fewer allowed than alternatives."""
    rng = np.random.default_rng(5)
    z = rng.standard_normal((rows, 1500)) * 2
    z[:, 300:900] = NEG
    z[0] = NEG
    z[1] = NEG
    z[1, 777] = -4.0
    z[2, 3:] = NEG
    z[5, :] = NEG
    z[5, 1499] = 1e30 if not bf16 else 1000.0
    p = Problem(torch, 6, rows, 1500, bf16, 10, z=z)
    p.tokens[0], p.tokens[1], p.tokens[2], p.tokens[3] = 4, 777, 1, 400
    both(p)
    assert p.logprob[0].item() == NEG and p.entropy[0].item() == 0 and (p.d[0] == 0).all() and p.top_id[0].tolist() == list(range(10))
    assert p.logprob[1].item() == 0 and p.logprob[3].item() == NEG


@pytest.mark.parametrize("scale", [1.0, 3.0])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,cols", [(6, 900), (2, 40000)])
def test_rows_of_the_lowest_value(torch, rows, cols, bf16, scale):
    """A mask of the type's lowest value on everything leaves the row uniform; on a part of it, nothing of that part."""
    low = -3.3895313892515355e38 if bf16 else -3.4028234663852886e38
    z = np.random.default_rng(7).standard_normal((rows, cols))
    z[0] = low
    z[1, 5:] = low
    p = Problem(torch, 8, rows, cols, bf16, 4, scale, z=z)
    p.tokens[0] = 9
    both(p)
    assert abs(p.entropy[0].item() - np.log(cols)) < 1e-5 and p.top_id[0].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("cols", [1000, 30000])
def test_not_a_number_stays_in_its_row(torch, cols):
    rows = 8
    z = np.random.default_rng(9).standard_normal((rows, cols))
    p = Problem(torch, 10, rows, cols, False, 3, z=z)
    both(p)
    keep = [t.clone() for t in (p.logprob, p.entropy, p.top_id, p.top_logprob, p.d)]
    p.z[2, 17] = float("nan")
    p.z[4, 18] = float("inf")
    p.tokens[2], p.tokens[4] = 1, 1
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    rest = [0, 1, 3, 5, 6, 7]
    for t, k in zip((p.logprob, p.entropy, p.top_id, p.top_logprob, p.d), keep):
        assert torch.equal(t[rest], k[rest])
    for r in (2, 4):
        assert p.logprob[r].isnan() and p.entropy[r].isnan() and p.top_logprob[r].isnan().all() and p.d[r].isnan().all()
    assert 17 not in p.top_id[2].tolist() and p.top_id[4, 0].item() == 18


def test_nothing_but_nan(torch):
    p = Problem(torch, 10, 2, 70, False, 5, z=np.full((2, 70), np.nan))
    p.forward()
    torch.cuda.synchronize()
    assert p.top_logprob.isnan().all() and (p.top_id == -1).all() and p.entropy.isnan().all()


@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "few values"])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,cols,top", [(3, 20000, 20), (700, 3001, 64)])
def test_alternatives_in_any_order(torch, rows, cols, top, order, bf16):
    """Rows in which every element, or none after the first, is among the best so far; ties, which go to the lower index."""
    rng = np.random.default_rng(11)
    z = {"ascending": np.linspace(-5, 5, cols), "descending": np.linspace(5, -5, cols), "equal": np.full(cols, 0.25),
         "few values": rng.integers(0, 4, cols).astype(float)}[order]
    z = np.broadcast_to(z, (rows, cols)).copy()
    if order == "few values":
        z[:, ::7] = -0.0        # equal to 0
    p = Problem(torch, 12, rows, cols, bf16, top, z=z)
    p.forward()
    p.check_forward()


def test_only_what_is_wanted(torch):
    p = Problem(torch, 13, 5, 700, top=3)
    both(p)
    want = {k: getattr(p, k).clone() for k in ("logprob", "entropy", "stats", "top_id")}
    none = dict(tokens=None, logprob=None, entropy=None, stats=None)
    p.top_id.fill_(0)
    p.forward(**none)
    torch.cuda.synchronize()
    assert torch.equal(p.top_id, want["top_id"])
    p.top = 0
    for name in ("entropy", "stats", "logprob"):
        getattr(p, name).fill_(0)
        p.forward(**{k: v for k, v in none.items() if k != name and not (name == "logprob" and k == "tokens")})
        torch.cuda.synchronize()
        assert torch.equal(getattr(p, name), want[name]), name
    p.backward(dentropy=None, entropy=None)
    p.check_backward(dentropy=False)
    p.backward(dlogprob=None, tokens=None)
    p.check_backward(dlogprob=False)


@pytest.mark.parametrize("rows,cols,pad", [(6, 5000, 0), (700, 1001, 3)])
def test_gradient_in_place(torch, rows, cols, pad):
    p = Problem(torch, 14, rows, cols, pad=pad)
    both(p)
    z = p.z.clone()
    p.backward(d=p.z)
    torch.cuda.synchronize()
    assert torch.equal(p.z, p.d) and not torch.equal(p.z, z)


@pytest.mark.parametrize("rows,cols", [(4, 51200), (900, 2500)])
def test_streams_graphs_and_repeats(torch, rows, cols):
    p, q = (Problem(torch, 15 + k, rows, cols, top=10) for k in range(2))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for a, s in zip((p, q), streams):
            a.forward(stream=s)
            a.backward(stream=s)
    for a in (p, q):
        a.check_forward()
        a.check_backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        with torch.cuda.graph(graph, stream=streams[0]):
            p.forward(stream=streams[0])
            p.backward(stream=streams[0])
    rng = np.random.default_rng(17)
    for _ in range(4):
        p.z.copy_(torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)))
        p.ws.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        p.check_forward()
        p.check_backward()
        first = [t.clone() for t in (p.logprob, p.entropy, p.d)]
        p.forward()
        p.backward()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (p.logprob, p.entropy, p.d)))


def test_a_small_workspace_is_refused(torch):
    p = Problem(torch, 18, 2, 100000, top=20)
    if p.ws_bytes:
        p.ws_bytes -= 1
        with pytest.raises(AssertionError):
            p.forward()
        torch.cuda.synchronize()
        assert (p.logprob == 7).all()


def test_offsets_beyond_32_bits(torch):
    rows, cols, ld = 1030, 100, 4200000
    p = Problem(torch, 19, rows, cols, top=3)
    both(p)
    wide = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    wide[:, :cols] = p.z
    p.z, p.d = wide[:, :cols], wide[:, cols:2 * cols]
    p.forward()
    p.backward()
    p.check_forward()       # (not the same bits: rows on other boundaries are added up in another order)
    p.check_backward()


def test_no_workspace_where_none_is_needed(torch):
    p = Problem(torch, 20, 70, 1500, top=4)
    assert p.ws_bytes == 0
    p.ws = None
    both(p)
    e = Problem(torch, 21, 0, 1500)
    e.ws = e.flat = e.z = None
    fn = K.lib()
    q = e.q(None)
    assert fn.karma_k_token_logprob_fwd_bf16(None, C.c_uint64(0), ptr(p.tokens), ptr(p.logprob), None, None, None, None, 0, 1500, 0, C.c_float(1), None,
                                             C.c_uint64(0), q) == K.OK
    assert fn.karma_k_token_logprob_bwd_bf16(None, C.c_uint64(0), ptr(p.tokens), None, None, ptr(p.dlogprob), None, None, C.c_uint64(0), 0, 1500,
                                             C.c_float(1), q) == K.OK
    p.check_forward()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("scale,weight,spread", [(1e10, 0.1, 3.0), (1e20, 1.0, 3.0), (1e19, 1.0, 3.0), (1.0, 1e9, 3.0), (1.0, 65536.0 * 1e30, 3.0),
                                                 (1e-20, 1.0, 3.0), (1e20, 1.0, 1e-20), (1e20, 1e15, 1e-20)])
@pytest.mark.parametrize("rows,cols", [(7, 900), (2, 30000)])
def test_entropy_gradient_where_scale_times_gradient_is_large(torch, rows, cols, scale, weight, spread, bf16):
    """A column that is not allowed, or whose probability is nothing, has no gradient, whatever the entropy's is."""
    z = np.random.default_rng(22).standard_normal((rows, cols)) * spread
    z[:, 100:300] = NEG
    z[0, 1:] = NEG
    p = Problem(torch, 23, rows, cols, bf16, scale=scale, z=z)
    p.dentropy.mul_(weight)
    p.forward()
    p.backward()
    p.check_backward()
    assert (p.d[:, 150:250].masked_fill((p.tokens[:, None] >= 150) & (p.tokens[:, None] < 250), 0) == 0).all()
    p.backward(dlogprob=None, tokens=None)
    p.check_backward(dlogprob=False)
    assert (p.d[:, 100:300] == 0).all()
