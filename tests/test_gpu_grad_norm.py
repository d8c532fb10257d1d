"""The global norm of gradients and clipping against the plain form in 64 bits: types, sizes, places off 16-byte boundaries, long lists, extremes,
with the AdamW step that takes the factor, and in a graph."""
import ctypes as C
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import decoder_forms as D
import paper_2008_11421_amd as K

U = D.U


class List:
    def __init__(self, tensors, outs=None, types=None):
        import torch
        self.g, self.out = tensors, outs or [None] * len(tensors)
        flags = lambda g, o: (K.GRAD_BF16 if g.dtype == torch.bfloat16 else 0) | (K.GRAD_OUT_BF16 if o is not None and o.dtype == torch.bfloat16 else 0)
        self.t = (K.GradTensor * len(tensors))(*[
            K.GradTensor(grad=g.data_ptr() if g.numel() else None, out=o.data_ptr() if o is not None and o.numel() else None, n=g.numel(), flags=flags(g, o))
            for g, o in zip(tensors, self.out)])
        self.ws = torch.full((max(16, K.grad_norm_ws_bytes(self.t)),), 255, dtype=torch.uint8, device="cuda")
        self.norm, self.factor = (torch.full((1,), 9.0, device="cuda") for _ in range(2))
        self.each = torch.full((len(tensors) + 1,), 9.0, device="cuda")

    def run(self, max_norm=1.0, scale=1.0, each=True, norm=True, factor=None):
        import gpu_util as g
        return K.lib().karma_k_grad_norm(self.t, len(self.t), C.c_float(max_norm), C.c_float(scale), g.ptr(self.norm) if norm else None,
                                         g.ptr(self.each) if each else None, factor or g.ptr(self.factor), g.ptr(self.ws), C.c_uint64(self.ws.numel()),
                                         g.stream_ptr())

    def clip(self):
        import gpu_util as g
        return K.lib().karma_k_grad_clip(self.t, len(self.t), g.ptr(self.factor), g.stream_ptr())

    def check(self, max_norm=1.0, scale=1.0):
        import torch
        torch.cuda.synchronize()
        norm, factor, each = D.grad_norm([g.double().cpu().numpy() for g in self.g], max_norm, scale)
        # 64 bits but for the rounding of the result
        near = lambda got, want: abs(got - want) <= (U + 1e-12) * abs(want) + 1e-45
        assert near(self.norm.item(), norm) and near(self.factor.item(), factor)
        got = self.each.cpu().numpy().astype(np.float64)
        assert got[-1] == 9.0 and all(near(a, b) for a, b in zip(got, each))
        return norm


def make(sizes, seed=0, types=("bf16", "f32"), off=(0,), std=1.0):
    import torch
    rng = np.random.default_rng(seed)
    T = {"bf16": torch.bfloat16, "f32": torch.float32}
    out = []
    for k, n in enumerate(sizes):
        o = off[k % len(off)]
        b = torch.from_numpy((std * rng.standard_normal(n + o)).astype(np.float32)).to(T[types[k % len(types)]]).cuda()
        out.append(b[o:])
    return out


@pytest.mark.parametrize("types", [("bf16",), ("f32",), ("bf16", "f32")])
@pytest.mark.parametrize("off", [(0,), (1, 3, 0, 7, 5)])
def test_sizes_and_places(types, off):
    import torch
    sizes = [0, 1, 2, 3, 7, 8, 9, 15, 16, 17, 63, 0, 255, 1000, 4095, 4096, 4097, 16383, 16385, 70001, 1]
    g = make(sizes, 1, types, off)
    keep = [t.clone() for t in g]
    a = List(g)
    assert a.run(3.0, 0.25) == 0
    a.check(3.0, 0.25)
    assert all(torch.equal(x, y) for x, y in zip(g, keep))
    for out_type in (torch.bfloat16, torch.float32):
        for shift in (0, 1, 4):
            room = [torch.full((n + 16,), 7.0, dtype=out_type, device="cuda") for n in sizes]
            outs = [r[shift:shift + n] for r, n in zip(room, sizes)]
            b = List(g, outs)
            assert b.run(3.0, 0.25) == 0 and b.clip() == 0
            b.check(3.0, 0.25)
            f = b.factor.double().item()
            for t, o, r, n in zip(g, outs, room, sizes):
                want = t.double() * f
                step = torch.finfo(out_type).eps / 2
                # a rounding of the product in 32 bits, and one to the result's type
                assert ((o.double() - want).abs() <= (step + U) * (1 + U) * want.abs() + 1e-40).all()
                assert (r[:shift] == 7).all() and (r[shift + n:] == 7).all()


def test_in_place_and_a_factor_of_one():
    import torch
    for types in (("bf16",), ("f32",)):
        g = make([100, 4097, 33], 2, types, (1, 0))
        keep = [t.clone() for t in g]
        a = List(g, g)
        assert a.run(1e6) == 0 and a.clip() == 0
        torch.cuda.synchronize()
        assert a.factor.item() == 1.0 and all(torch.equal(x, y) for x, y in zip(g, keep))
        assert a.run(2.0) == 0 and a.clip() == 0
        torch.cuda.synchronize()
        f = a.factor
        assert all(torch.equal(x, (y.float() * f).to(x.dtype)) for x, y in zip(g, keep))
        b = List(g)
        assert b.run(2.0) == 0
        torch.cuda.synchronize()
        # half a step of every element, at most
        assert abs(b.norm.item() - 2.0) <= 2 * 2.0 * torch.finfo(g[0].dtype).eps / 2


def test_long_lists():
    import torch
    sizes = [(k * 37) % 301 for k in range(2111)]
    sizes[5], sizes[1500] = 100000, 33333
    g = make(sizes, 3)
    outs = [torch.zeros_like(t) for t in g]
    a = List(g, outs)
    assert a.run(5.0, 2.0) == 0 and a.clip() == 0
    a.check(5.0, 2.0)
    assert all(torch.equal(o, (t.float() * a.factor).to(t.dtype)) for o, t in zip(outs, g))


def test_large_tensors():
    import torch
    g = make([17_000_001, 1_234_567], 4, ("bf16", "f32"), (3, 1))
    a = List(g)
    assert a.run(1.0) == 0
    a.check(1.0)


def test_empty_lists():
    import torch
    import gpu_util as g
    a = List(make([0, 0], 1))
    assert a.run(1.0, 0.5) == 0
    torch.cuda.synchronize()
    assert a.norm.item() == 0 and a.factor.item() == 0.5 and a.each[:2].tolist() == [0, 0]
    ws = torch.zeros(16, dtype=torch.uint8, device="cuda")
    assert K.lib().karma_k_grad_norm(None, 0, C.c_float(1.0), C.c_float(2.0), g.ptr(a.norm), g.ptr(a.each), g.ptr(a.factor), g.ptr(ws), C.c_uint64(16),
                                     g.stream_ptr()) == 0
    torch.cuda.synchronize()
    assert a.factor.item() == 2.0 and a.clip() == 0


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_extremes(t):
    """Squares that 32 bits do not hold, and values that are no numbers."""
    import torch
    for std in (1e30, 1e-30):
        a = List(make([5000, 77], 5, (t,), (1,), std))
        assert a.run(1.0) == 0
        a.check(1.0)
    g = make([1000, 50], 6, (t,))
    a = List(g)
    assert a.run(math.inf, 0.5) == 0
    a.check(math.inf, 0.5)
    assert a.factor.item() == 0.5
    g[1][7] = -math.inf
    assert a.run(1.0) == 0
    torch.cuda.synchronize()
    assert a.norm.item() == math.inf and a.factor.item() == 0 and a.each[1].item() == math.inf and math.isfinite(a.each[0].item())
    g[0][999] = math.nan
    assert a.run(1.0) == 0
    torch.cuda.synchronize()
    assert math.isnan(a.norm.item()) and math.isnan(a.factor.item()) and math.isnan(a.each[0].item()) and a.each[1].item() == math.inf


def test_each_output_alone():
    import torch
    a = List(make([1000, 50], 7))
    assert a.run() == 0
    want = a.norm.clone(), a.factor.clone(), a.each.clone()
    for k in range(3):
        b = List(a.g)
        import gpu_util as g
        ptr = lambda j, t: g.ptr(t) if j == k else None
        assert K.lib().karma_k_grad_norm(b.t, 2, C.c_float(1.0), C.c_float(1.0), ptr(0, b.norm), ptr(1, b.each), ptr(2, b.factor), g.ptr(b.ws),
                                         C.c_uint64(b.ws.numel()), g.stream_ptr()) == 0
        torch.cuda.synchronize()
        for j, (got, w) in enumerate(zip((b.norm, b.factor, b.each), (want[0], want[1], want[2]))):
            place = {0: 0, 1: 2, 2: 1}[j]
            assert torch.equal(got, w) if place == k else (got == 9.0).all()


def test_the_update_takes_the_factor():
    """The factor goes into the AdamW step's live values: the same update as with clipped gradients."""
    import torch
    import gpu_util as g
    sizes = [4097, 100, 33]
    grads = make(sizes, 8, ("f32",))
    start = make(sizes, 9, ("f32",))
    live = torch.zeros(4, device="cuda")
    live[0] = 1e-3
    live.view(torch.int32)[2] = 1       # the step
    a = List(grads)
    assert a.run(1.0, 0.5, factor=C.c_void_p(live.data_ptr() + 4)) == 0
    now = K.AdamwStep(lr=9.0, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=9.0, seed=0, step=9)
    w, m, v = [t.clone() for t in start], [torch.zeros_like(t) for t in start], [torch.zeros_like(t) for t in start]
    ts = (K.AdamwTensor * 3)(*[K.AdamwTensor(w=w[k].data_ptr(), m=m[k].data_ptr(), v=v[k].data_ptr(), grad=grads[k].data_ptr(), n=sizes[k], weight_decay=0.1)
                               for k in range(3)])
    assert K.lib().karma_k_adamw(ts, 3, C.byref(now), g.ptr(live), g.stream_ptr()) == 0
    torch.cuda.synchronize()
    norm, factor, _ = D.grad_norm([t.double().cpu().numpy() for t in grads], 1.0, 0.5)
    assert norm > 1.0 and abs(live[1].item() - factor) <= U * factor
    import operator_forms as F
    for k in range(3):
        want, wm, _ = F.adamw(start[k].cpu().numpy(), 0, 0, grads[k].cpu().numpy(), 0.1, 1e-3, 0.9, 0.95, 1e-8, live[1].item(), 1)
        # |w| < 8: a rounding of it, the update is 1e-3
        assert np.abs(w[k].cpu().numpy() - want).max() <= 2 * U * 8
        assert np.abs(m[k].cpu().numpy() - wm).max() <= 8 * U * np.abs(wm).max()


def test_on_another_stream_and_in_two_graphs():
    import torch
    g = make([5000, 77, 70001], 10, off=(1, 0))
    a = List(g, [torch.zeros_like(t) for t in g])
    assert a.run(2.0) == 0 and a.clip() == 0
    torch.cuda.synchronize()
    lists = [List(g, [torch.zeros_like(t) for t in g]) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert lists[0].run(2.0) == 0 and lists[0].clip() == 0
    side.synchronize()
    same = lambda b: torch.equal(a.norm, b.norm) and torch.equal(a.factor, b.factor) and torch.equal(a.each, b.each) and all(
        torch.equal(x, y) for x, y in zip(a.out, b.out))
    assert same(lists[0])
    graphs = []
    for b in lists:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            assert b.run(2.0) == 0 and b.clip() == 0
        graphs.append(gr)
    for _ in range(3):
        for b in lists:
            for t in (b.norm, b.factor, b.each[:3], *b.out):
                t.fill_(5.0)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(same(b) for b in lists)


def test_a_tensor_beyond_32_bits():
    import torch
    n = (1 << 31) + 1001
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[1 << 31] = 300.0, -200.0
    out = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    a = List([g], [out])
    assert a.run(1.0) == 0 and a.clip() == 0
    torch.cuda.synchronize()
    want = math.sqrt(n - 2 + 300.0 ** 2 + 200.0 ** 2)
    assert abs(a.norm.item() - want) <= (U + 1e-12) * want and a.each[0].item() == a.norm.item()
    f = a.factor
    for i in (0, 1 << 20, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, n - 2, n - 1):
        assert torch.equal(out[i], (g[i].float() * f[0]).to(torch.bfloat16)), i
    assert int((out == (f[0]).to(torch.bfloat16)).sum()) == n - 2


def test_two_calls_at_once():
    import torch
    lists = [List(g, [torch.zeros_like(t) for t in g]) for g in (make([70001, 5000, 33], 11), make([123456, 77], 12, ("f32",)))]
    want = []
    for a in lists:
        assert a.run(2.0) == 0 and a.clip() == 0
        torch.cuda.synchronize()
        want.append([t.clone() for t in (a.norm, a.factor, a.each, *a.out)])
        for t in (a.norm, a.factor, *a.out):
            t.zero_()
    streams = [torch.cuda.Stream() for _ in lists]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, s in zip(lists, streams):
            with torch.cuda.stream(s):
                assert a.run(2.0) == 0 and a.clip() == 0
    torch.cuda.synchronize()
    for a, w in zip(lists, want):
        assert all(torch.equal(x, y) for x, y in zip((a.norm, a.factor, a.each, *a.out), w))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1])
def test_clipping_and_updates_of_values_that_are_no_numbers(t, off):
    """What an infinite norm leaves: a factor of 0, under which infinite values become NaN and all others 0; NaN spoils all."""
    import torch
    import gpu_util as gu
    for out in (torch.bfloat16, torch.float32):
        g = make([1000, 4099], 13, (t,), (off,))
        g[0][7], g[0][999], g[1][4098], g[1][64] = math.inf, -math.inf, math.inf, -math.inf
        a = List(g, [torch.full_like(x, 5.0, dtype=out) for x in g])
        assert a.run(1.0) == 0 and a.clip() == 0
        torch.cuda.synchronize()
        assert a.norm.item() == math.inf and a.factor.item() == 0
        for x, o in zip(g, a.out):
            assert torch.isnan(o[torch.isinf(x)]).all() and (o[torch.isfinite(x)] == 0).all()
        # the update that takes the factor: the same values' weights and states
        live = torch.zeros(4, device="cuda")
        live[0], live[1] = 1e-3, a.factor[0]
        live.view(torch.int32)[2] = 1
        now = K.AdamwStep(lr=9.0, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=9.0, seed=0, step=9)
        w, m, v = [torch.ones(x.numel(), device="cuda") for x in g], [torch.zeros(x.numel(), device="cuda") for x in g], [torch.zeros(x.numel(), device="cuda") for x in g]
        ts = (K.AdamwTensor * 2)(*[K.AdamwTensor(w=w[k].data_ptr(), m=m[k].data_ptr(), v=v[k].data_ptr(), grad=g[k].data_ptr(), n=g[k].numel(),
                                                 flags=K.ADAMW_GRAD_BF16 if t == "bf16" else 0) for k in range(2)])
        assert K.lib().karma_k_adamw(ts, 2, C.byref(now), gu.ptr(live), gu.stream_ptr()) == 0
        torch.cuda.synchronize()
        for k, x in enumerate(g):
            bad = torch.isinf(x)
            for s in (w[k], m[k], v[k]):
                assert torch.isnan(s[bad]).all() and torch.isfinite(s[~bad]).all()
        g[0][500] = math.nan
        assert a.run(1.0) == 0 and a.clip() == 0
        torch.cuda.synchronize()
        assert math.isnan(a.norm.item()) and math.isnan(a.factor.item()) and all(torch.isnan(o).all() for o in a.out)
