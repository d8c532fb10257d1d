"""The AdamW step over many tensors on the GPU against its form in 64 bits: types, 32 and 8-bit states, sizes, alignments, and
the ways it is called."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import operator_forms as F
import paper_2008_11421_amd as K


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


class Live(C.Structure):
    _fields_ = [("lr", C.c_float), ("grad_scale", C.c_float), ("step", C.c_uint32), ("seed", C.c_uint32)]


class Step:
    """A list of tensors: (size, gradient in bf16, out None / "bf16" / "f32", 8 bits, weight decay), each buffer `lead` elements into
    its allocation."""

    def __init__(self, torch, seed, specs, lead=0, lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=0.7, step=7, rseed=99):
        self.torch, self.specs = torch, specs
        self.hyper = dict(lr=lr, beta1=beta1, beta2=beta2, eps=eps, grad_scale=grad_scale, step=step, seed=rseed)
        rng = np.random.default_rng(seed)
        put = lambda a, t: self._put(a, t, lead)
        self.w, self.g, self.out, self.m, self.v, self.ms, self.vs = [], [], [], [], [], [], []
        for n, gbf, out, eight, _ in specs:
            blocks = -(-n // 64)
            self.w.append(put(rng.standard_normal(n), torch.float32))
            self.g.append(put(rng.standard_normal(n) * np.exp(rng.standard_normal(n)), torch.bfloat16 if gbf else torch.float32))
            self.out.append(put(np.full(n, 7.0), torch.bfloat16 if out == "bf16" else torch.float32) if out else None)
            if eight:
                self.m.append(put(rng.integers(-127, 128, n), torch.int8))
                self.v.append(put(rng.integers(0, 256, n), torch.uint8))
                self.ms.append(put(rng.random(blocks) * 1e-3, torch.float32))
                self.vs.append(put(rng.random(blocks) * 1e-6, torch.float32))
            else:
                self.m.append(put(rng.standard_normal(n) * 0.1, torch.float32))
                self.v.append(put(rng.random(n) * 0.01, torch.float32))
                self.ms.append(None)
                self.vs.append(None)

    def _put(self, a, t, lead):
        flat = self.torch.full((lead + len(a) + 8,), 9, dtype=t, device="cuda")
        flat[lead:lead + len(a)] = self.torch.from_numpy(np.asarray(a, np.float32)).to(t).cuda()
        return flat[lead:lead + len(a)]

    def tensors(self):
        p = lambda t: t.data_ptr() if t is not None else None
        return (K.AdamwTensor * len(self.specs))(*[
            K.AdamwTensor(w=p(self.w[k]), m=p(self.m[k]), v=p(self.v[k]), m_scale=p(self.ms[k]), v_scale=p(self.vs[k]), grad=p(self.g[k]),
                          out=p(self.out[k]), n=n, weight_decay=decay,
                          flags=(1 if gbf else 0) | (2 if out == "bf16" else 0) | (4 if eight else 0))
            for k, (n, gbf, out, eight, decay) in enumerate(self.specs)])

    def run(self, stream=None, live=None, **change):
        q = C.c_void_p((stream or self.torch.cuda.current_stream()).cuda_stream)
        now = K.AdamwStep(**{**self.hyper, **change})
        st = K.lib().karma_k_adamw(self.tensors(), len(self.specs), C.byref(now), C.c_void_p(live.data_ptr()) if live is not None else None, q)
        assert st == K.OK, st

    def values(self):
        """(m, v) of every tensor in 64 bits, from what is stored"""
        h = lambda t: t.cpu().numpy()
        m, v = [], []
        for k, (n, _, _, eight, _) in enumerate(self.specs):
            a, b = h(self.m[k]).astype(np.float64), h(self.v[k]).astype(np.float64)
            if eight:
                a, b = a * F.by_block(h(self.ms[k]), n), b * b * F.by_block(h(self.vs[k]), n)
            m.append(a)
            v.append(b)
        return m, v

    def check(self, change=None):
        """Runs a step and compares everything it wrote."""
        h = lambda t: t.float().cpu().numpy()
        self.torch.cuda.synchronize()
        w0, g0, (m0, v0) = [h(t) for t in self.w], [h(t) for t in self.g], self.values()
        hy = {**self.hyper, **(change or {})}
        self.run(**(change or {}))
        self.compare(w0, g0, m0, v0, hy)

    def compare(self, w0, g0, m0, v0, hy):
        h = lambda t: t.float().cpu().numpy()
        self.torch.cuda.synchronize()
        b1, b2, gs = F.f32(hy["beta1"]), F.f32(hy["beta2"]), F.f32(hy["grad_scale"])
        U = F.U
        for k, (n, gbf, out, eight, decay) in enumerate(self.specs):
            w, m, v = F.adamw(w0[k], m0[k], v0[k], g0[k], decay, hy["lr"], hy["beta1"], hy["beta2"], hy["eps"], hy["grad_scale"], hy["step"])
            got = h(self.w[k]).astype(np.float64)
            # the moments: each term is off by the roundings of its factors and products, and the sum by one
            em = (6 * U) * (b1 * np.abs(m0[k]) + (1 - b1) * np.abs(gs * g0[k]))
            ev = (8 * U) * (b2 * v0[k] + (1 - b2) * (gs * g0[k].astype(np.float64)) ** 2)
            if eight:
                em, ev = np.abs(m) * U * 2, v * U * 2           # computed in 64 bits, rounded once for the update
            c1, c2 = 1 / (1 - b1 ** hy["step"]), 1 / (1 - b2 ** hy["step"])
            den = np.sqrt(v * c2) + F.f32(hy["eps"])
            up = c1 * np.abs(m) / den
            lr = F.f32(hy["lr"])
            # the update: root, product, sum, quotient and products, 2 U each where they are not a rounding alone; w: decay and two sums
            eup = lr * (c1 * em / den + up * (ev / np.maximum(2 * v, 1e-300) + 14 * U))
            bound = eup + U * (3 * np.abs(w0[k]) * (1 + lr * decay) + 2 * lr * up) + 1e-38
            assert (np.abs(got - w) <= bound).all(), (k, np.abs(got - w).max(), bound[np.abs(got - w).argmax()])
            if out:
                assert np.array_equal(h(self.out[k]), h(self.w[k].to(self.torch.bfloat16 if out == "bf16" else self.torch.float32)))
            if not eight:
                assert (np.abs(h(self.m[k]) - m) <= em).all() and (np.abs(h(self.v[k]) - v) <= ev).all(), k
            else:
                cm, sm, cv, sv = F.quantised(m, v, k, hy["seed"])
                assert np.array_equal(self.ms[k].cpu().numpy(), sm) and np.array_equal(self.vs[k].cpu().numpy(), sv), k
                assert np.array_equal(self.m[k].cpu().numpy(), cm), (k, np.flatnonzero(self.m[k].cpu().numpy() != cm)[:5])
                assert np.array_equal(self.v[k].cpu().numpy(), cv), (k, np.flatnonzero(self.v[k].cpu().numpy() != cv)[:5])
            for t in (self.w[k], self.m[k], self.v[k], self.out[k], self.ms[k], self.vs[k]):
                if t is not None:       # what lies behind a tensor is not its own
                    assert (self.torch.as_strided(t, (8,), (1,), t.storage_offset() + t.numel()) == 9).all()


SIZES = [1, 2, 3, 5, 63, 64, 65, 127, 128, 255, 256, 257, 1000, 1023, 1024, 1025, 4095, 4096, 4097, 16384, 16387, 70001]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("gbf,out", [(True, "bf16"), (False, "f32"), (True, None), (False, "bf16"), (True, "f32")])
def test_sizes_and_types(torch, gbf, out, eight):
    s = Step(torch, 1, [(n, gbf, out, eight, 0.1 * (k % 3)) for k, n in enumerate(SIZES)])
    s.check()
    s.check(dict(step=8, seed=100))


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lead", [1, 2, 3, 5])
def test_alignment(torch, lead, eight):
    Step(torch, 2, [(n, True, "bf16", eight, 0.1) for n in (1, 63, 64, 300, 5000)], lead=lead).check()
    Step(torch, 2, [(n, False, "f32", eight, 0.1) for n in (1, 63, 64, 300, 5000)], lead=lead).check()


def test_many_tensors_of_all_kinds(torch):
    rng = np.random.default_rng(3)
    specs = [(int(rng.integers(0, 3000)), bool(rng.integers(2)), [None, "bf16", "f32"][rng.integers(3)], bool(rng.integers(2)), float(rng.random()))
             for _ in range(300)]
    specs[7] = specs[150] = (0, True, None, True, 0.0)
    Step(torch, 3, specs).check()


def test_a_large_tensor(torch):
    s = Step(torch, 4, [(3, True, None, False, 0.0), (5_000_003, True, "bf16", True, 0.1), (3_000_001, False, "bf16", False, 0.1)])
    s.check()


def test_states_at_the_beginning(torch):
    s = Step(torch, 5, [(1000, True, "bf16", True, 0.0), (1000, True, "bf16", False, 0.0)], step=1, grad_scale=1.0)
    for ts in (s.m, s.v, s.ms, s.vs):
        for t in ts:
            if t is not None:
                t.zero_()
    s.g[0][64:256] = 0          # blocks that stay at zero
    s.check()
    assert (s.ms[0][1:4] == 0).all() and (s.m[0][64:256] == 0).all()
    # and no state rounds to a second moment of zero beside a first one
    s.check(dict(step=2, seed=3))
    assert ((s.v[0] > 0) | (s.m[0] == 0)).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_gradients_that_are_not_finite(torch, bad):
    s = Step(torch, 6, [(256, False, None, True, 0.0), (256, False, None, False, 0.0)])
    s.g[0][70], s.g[1][70] = bad, bad
    s.run()
    torch.cuda.synchronize()
    (m8, m32), (v8, v32) = s.values()
    lost = np.zeros(256, bool)
    lost[64:128] = True
    assert np.array_equal(np.isnan(m8), lost) and np.array_equal(np.isnan(v8), lost)
    one = np.zeros(256, bool)
    one[70] = True
    assert np.array_equal(~np.isfinite(m32), one)
    # the step itself is lost for the one weight alone
    assert np.array_equal(~np.isfinite(s.w[0].cpu().numpy()), one) and np.array_equal(~np.isfinite(s.w[1].cpu().numpy()), one)


def test_weight_decay_alone_and_no_learning(torch):
    s = Step(torch, 7, [(500, True, None, False, 0.5)], grad_scale=0.0)
    s.m[0].zero_()
    w = s.w[0].clone()
    s.check()
    assert not torch.equal(w, s.w[0])
    s = Step(torch, 7, [(500, True, "f32", True, 0.5)], lr=0.0)
    w = s.w[0].clone()
    s.check()
    assert torch.equal(w, s.w[0])


def test_a_small_decay_is_rounded_once(torch):
    """lr * decay = 0.6 * 2^-24 takes 0.45 of a step (2^-23) off 1.5: the nearest number is 1.5.  Rounded by itself, 1 - lr * decay would be
    1 - 2^-24, and 1.5 times that nearest to 1.5 - 2^-23.  At 0.7 * 2^-24 it is 0.525 of a step."""
    for share, want in ((0.6, 1.5), (0.7, 1.5 - 2.0 ** -23)):
        s = Step(torch, 7, [(256, False, None, False, share)], lr=2.0 ** -24, beta1=0.0, beta2=0.0, eps=1.0)
        s.w[0].fill_(1.5)
        s.g[0].zero_()
        s.run()
        torch.cuda.synchronize()
        assert (s.w[0] == want).all()


@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 6, 2 ** 40])
def test_step_numbers(torch, step):
    Step(torch, 8, [(300, True, None, False, 0.1), (300, True, None, True, 0.1)], step=step, beta2=0.999).check()


@pytest.mark.parametrize("betas", [(0.0, 0.0), (0.0, 0.999), (0.95, 0.0)])
def test_betas(torch, betas):
    Step(torch, 9, [(300, True, None, False, 0.1), (300, True, None, True, 0.1)], beta1=betas[0], beta2=betas[1], eps=1e-3).check()


def test_states_as_values(torch):
    s = Step(torch, 10, [(n, True, None, True, 0.0) for n in (1, 64, 100, 5001, 0, 70000)] * 10)
    outs = [[torch.full((n + 8,), 9.0, device="cuda") for n, *_ in s.specs] for _ in range(2)]
    arr = [(C.c_void_p * len(s.specs))(*[t.data_ptr() for t in o]) for o in outs]
    assert K.lib().karma_k_adamw_states(s.tensors(), len(s.specs), arr[0], arr[1], C.c_void_p(torch.cuda.current_stream().cuda_stream)) == K.OK
    torch.cuda.synchronize()
    for got, want in zip(outs, s.values()):
        for t, w, (n, *_) in zip(got, want, s.specs):
            assert (np.abs(t[:n].cpu().numpy() - w) <= F.U * np.abs(w) + 1e-45).all() and (t[n:] == 9).all()


def test_many_steps_follow_the_exact_moments(torch):
    """200 steps with noisy gradients: the 8-bit second moment stays near the exact one on average (rounding to the nearest code would
    leave it where it stalls, near 0.4 of it), and the weights move like those with 32-bit states."""
    n = 1 << 14
    s = Step(torch, 11, [(n, False, None, True, 0.0), (n, False, None, False, 0.0)], beta2=0.999, lr=1e-3, grad_scale=1.0)
    for ts in (s.m, s.v, s.ms, s.vs):
        for t in ts:
            if t is not None:
                t.zero_()
    s.w[1].copy_(s.w[0])
    w0 = s.w[0].clone()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for step in range(1, 201):
        s.g[0].normal_(0.2, 1.0, generator=gen)
        s.g[1].copy_(s.g[0])
        s.run(step=step, seed=step)
    torch.cuda.synchronize()
    (m8, m32), (v8, v32) = s.values()
    # unbiased codes: the mean over 16384 values is within a few parts in a thousand; the floor of code 1 adds less than that
    assert abs(v8.mean() / v32.mean() - 1) < 0.01
    d8, d32 = (s.w[0] - w0).double(), (s.w[1] - w0).double()
    assert float((d8 * d32).sum() / (d8.norm() * d32.norm())) > 0.99 and abs(float(d8.norm() / d32.norm()) - 1) < 0.02


def test_captured_step_reads_live_values(torch):
    specs = [(1000, True, "bf16", True, 0.1), (777, False, None, False, 0.1)]
    s = Step(torch, 12, specs)
    live = torch.zeros(4, dtype=torch.int32, device="cuda")

    def write(lr, gs, step, seed):
        live.copy_(torch.from_numpy(np.frombuffer(bytes(Live(lr, gs, step, seed)), dtype=np.int32).copy()))

    write(1e-2, 0.7, 1, 1)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s.run(stream=side, live=live, step=0, lr=float("nan"))      # not looked at
    h = lambda t: t.float().cpu().numpy()
    for k in range(4):
        hy = dict(s.hyper, lr=1e-3 * (k + 1), grad_scale=0.5 + k, step=k + 1, seed=11 * k + 2 ** 31)
        write(hy["lr"], hy["grad_scale"], hy["step"], hy["seed"])
        torch.cuda.synchronize()
        w0, g0, (m0, v0) = [h(t) for t in s.w], [h(t) for t in s.g], s.values()
        graph.replay()
        s.compare(w0, g0, m0, v0, hy)


def test_two_streams_at_once(torch):
    a, b = (Step(torch, 13 + k, [(9000, True, "bf16", bool(k), 0.1)] * 60) for k in range(2))
    h = lambda t: t.float().cpu().numpy()
    before = [([h(t) for t in s.w], [h(t) for t in s.g], *s.values()) for s in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, q in zip((a, b), streams):
        s.run(stream=q)
    torch.cuda.synchronize()
    for s, (w0, g0, m0, v0) in zip((a, b), before):
        s.compare(w0, g0, m0, v0, s.hyper)
