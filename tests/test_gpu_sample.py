"""Drawing tokens against the plain form in 64 bits: the same tokens and counts for every rule, also at borders, among equal logits, with masks, and the
right shares over all random numbers."""
import ctypes as C
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import decoder_forms as D
import paper_2008_11421_amd as K

U = D.U


def rules_of(rules):
    import torch
    a = np.zeros((len(rules), 4), np.float32)
    for k, (T, p, mp, top) in enumerate(rules):
        a[k, :3] = T, p, mp
        a[k, 3:].view(np.uint32)[0] = top
    return torch.from_numpy(a).cuda()


def workspace(rows, cols):
    import torch
    return torch.full((max(16, K.sample_ws_bytes(rows, cols)),), 255, dtype=torch.uint8, device="cuda")


def draw(z, rules, u, ld=0, cols=None, ws=None, outs=(1, 1, 1), stream=None):
    """z: a tensor [rows][ld] on the GPU; (token, logprob, kept)"""
    import torch
    import gpu_util as g
    rows, cols = z.shape[0], cols or z.shape[1]
    fn = K.lib().karma_k_sample_bf16 if z.dtype == torch.bfloat16 else K.lib().karma_k_sample_f32
    r = rules if isinstance(rules, torch.Tensor) else rules_of(rules)
    un = u if isinstance(u, torch.Tensor) else torch.tensor(np.asarray(u, np.float32), device="cuda")
    ws = workspace(rows, cols) if ws is None else ws
    token, kept = (torch.full((rows,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    logprob = torch.full((rows,), 77.0, device="cuda")
    p = lambda t, on: g.ptr(t) if on else None
    assert fn(g.ptr(z), C.c_uint64(z.stride(0) if rows > 1 else ld), g.ptr(r), r.shape[0], g.ptr(un), p(token, outs[0]), p(logprob, outs[1]), p(kept, outs[2]),
              rows, cols, g.ptr(ws), C.c_uint64(ws.numel()), stream or g.stream_ptr()) == 0
    torch.cuda.synchronize()
    return token.cpu().numpy(), logprob.cpu().numpy(), kept.cpu().numpy()


def check(z, rules, u, cols=None):
    token, logprob, kept = draw(z, rules, u, cols=cols)
    cols = cols or z.shape[1]
    h = z[:, :cols].double().cpu().numpy()
    f = lambda v: float(np.float32(v))
    for r in range(z.shape[0]):
        T, p, mp, top = rules[0 if len(rules) == 1 else r]
        want = D.sample_row(h[r], f(T), f(p), f(mp), top, f(u[r]))
        assert (token[r], kept[r]) == (want[0], want[2]), (r, rules[0 if len(rules) == 1 else r], u[r], want)
        if want[0] >= 0:
            # 64 bits and whole numbers but for the rounding of the result: weights are off by half of 2^-40
            assert abs(logprob[r] - want[1]) <= U * abs(want[1]) + 1e-9, r
        else:
            assert math.isnan(logprob[r])
    return token, logprob, kept


def types():
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}


RULES = [(1.0, 1.0, 0.0, 0), (0.7, 0.9, 0.0, 50), (1.0, 0.95, 0.0, 0), (1.3, 1.0, 0.05, 0), (1.0, 1.0, 0.0, 20), (0.8, 0.5, 0.1, 7), (0.0, 0.9, 0.0, 5),
         (1.0, 0.9, 0.0, 1), (1.0, 0.0, 0.0, 0), (2.0, 0.99999, 0.0, 0), (1.0, 1e-6, 0.0, 0), (1.0, 0.9, 1.0, 0), (1.0, 7.0, 9.0, 10 ** 9), (0.05, 0.999, 0.0, 100),
         (30.0, 0.5, 0.0, 1000), (1e-30, 0.9, 0.0, 3), (1e30, 0.3, 0.0, 0), (1.0, 0.9, -1.0, 2)]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1, 2, 7, 8, 9, 63, 500, 513, 1000, 8191, 32000, 50021])
def test_rules_and_sizes(t, cols):
    import torch
    rng = np.random.default_rng(cols)
    n = len(RULES)
    z = 2 * rng.standard_normal((n, cols)).astype(np.float32)
    z[:, rng.integers(0, cols, 5)] += 6
    z = torch.from_numpy(z).to(types()[t]).cuda()
    for u in (rng.random(n), np.zeros(n), np.full(n, 1 - 2.0 ** -24)):
        check(z, RULES, u.astype(np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [1, 3, 8])
def test_strides_and_places(t, extra):
    """Rows that begin anywhere; what lies behind a row's columns is not looked at."""
    import torch
    rng = np.random.default_rng(extra)
    n, cols = len(RULES), 1003
    room = torch.full((n * (cols + extra) + 16,), float("nan"), dtype=types()[t], device="cuda")
    z = room[extra:extra + n * (cols + extra)].view(n, cols + extra)
    z[:, :cols] = torch.from_numpy(3 * rng.standard_normal((n, cols)).astype(np.float32)).to(z.dtype).cuda()
    check(z, RULES, rng.random(n).astype(np.float32), cols=cols)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_equal_logits(t):
    """Of equal logits the first ones stay, however many there are."""
    import torch
    for cols in (8, 1024, 5000, 40000):
        rules = [(1.0, 0.5, 0.0, 0), (1.0, 1.0, 0.0, 3), (1.0, 0.25, 0.0, 2 + cols // 2), (0.5, 1.0, 1.0, 0), (1.0, 0.999, 0.0, cols - 1), (1.0, 1.0, 0.0, 0)]
        z = torch.full((len(rules), cols), 1.5, dtype=types()[t], device="cuda")
        for u in (0.0, 0.5, 0.99999):
            check(z, rules, np.full(len(rules), u, np.float32))
        z[:, cols // 3:] = 1.0          # two values, many of each
        z[:, 1::7] = -4.0
        for u in (0.0, 0.3, 0.99999):
            check(z, rules, np.full(len(rules), u, np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_many_values_close_together(t):
    """Logits that one bin holds, of both signs and next to zero: it is cut again by their bits."""
    import torch
    rng = np.random.default_rng(5)
    rules = [(1.0, 0.5, 0.0, 0), (1.0, 1.0, 0.0, 1234), (1.0, 0.3, 0.0, 20000), (100.0, 0.77, 0.0, 0), (1.0, 0.999, 0.0, 39999), (1.0, 0.001, 0.0, 17)]
    for width in (1e-2, 1e-5, 1e-30):
        z = torch.from_numpy((width * rng.standard_normal((len(rules), 40000))).astype(np.float32)).to(types()[t]).cuda()
        z[:, ::11] = 0.0
        z[:, 5::11] = -0.0
        check(z, rules, rng.random(len(rules)).astype(np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_numbers_of_every_size(t):
    """Rows with a few logits next to 0, far below or far above the others, and of one sign."""
    import torch
    rng = np.random.default_rng(12)
    rules = [(1.0, 0.9, 0.0, 0), (1.0, 1.0, 0.0, 300), (0.5, 0.5, 0.0, 0), (1.0, 0.999, 0.01, 0), (1e5, 0.7, 0.0, 0), (1e5, 1.0, 0.0, 600), (3.0, 0.99, 0.0, 700),
             (1.0, 1.0, 0.0, 0), (20.0, 0.6, 0.0, 0), (1.0, 0.9, 0.0, 20)]
    cols = 1200
    base = rng.standard_normal((len(rules), cols)).astype(np.float32)
    tiny = base.copy()
    at = rng.integers(0, cols, 12)
    tiny[:, at] = np.array([1e-5, -1e-5, 1e-6, -1e-6, 3e-5, -3e-5, 1e-20, -1e-20, 1e-40, 0.0, -0.0, 5e-5], np.float32)
    flat = np.where(np.abs(base) > 1.5, -base ** 2, 0).astype(np.float32)       # mostly zeros, the largest
    flat[:, at] = tiny[:, at]
    far = base.copy()
    far[:, ::5] = -1e6
    far[:, 1::50] = -3e5
    high = base.copy()
    high[:, 700] = 1e6
    high[:, 701] = 1e6
    for z in (tiny, flat, far, high, base - 9, base + 9, 1e-3 * base - 300000, 40 * base):
        z = torch.from_numpy(np.ascontiguousarray(z, np.float32)).to(types()[t]).cuda()
        for u in (rng.random(len(rules)), np.full(len(rules), 0.9999999)):
            check(z, rules, u.astype(np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_rows_for_every_number_of_threads(t):
    import torch
    rng = np.random.default_rng(13)
    for rows, cols in ((257, 13000), (257, 700), (3, 13000), (2, 9000), (2, 70001)):
        z = torch.from_numpy((2 * rng.standard_normal((rows, cols))).astype(np.float32)).to(types()[t]).cuda()
        rules = [RULES[r % len(RULES)] for r in range(rows)]
        for u in (rng.random(rows), np.full(rows, 0.999)):
            check(z, rules, u.astype(np.float32))
    z = torch.from_numpy((2 * rng.standard_normal((8, 140001))).astype(np.float32)).to(types()[t]).cuda()
    check(z, [(1.0, 0.9, 0.0, 0), (0.7, 0.95, 0.0, 40), (1.0, 1.0, 0.0, 0), (1.3, 0.97, 0.02, 0), (1.0, 0.9, 0.0, 96), (1.0, 0.9, 0.0, 129), (1.5, 1.0, 0.0, 5000),
              (0.8, 1.0, 0.1, 0)], rng.random(8).astype(np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_min_p_alone(t):
    """From next to nothing to the largest, at temperatures and places where few bits are left of the logits' differences."""
    import torch
    rng = np.random.default_rng(17)
    min_p = [1e-12, 2e-12, 3e-12, 1e-9, 1e-3, 0.05, 0.5, 0.999, 1.0]
    for T in (1e-3, 0.7, 1.0, 50.0, 1e30):
        for at in (0.0, 40.0, -3000.0, 2.0 ** 20):
            z = (at + 4 * max(T, 1e-2) * rng.standard_normal((len(min_p), 3000))).astype(np.float32)
            z = torch.from_numpy(z).clamp(-1e38, 1e38).to(types()[t]).cuda()
            check(z, [(T, 1.0, m, 0) for m in min_p], rng.random(len(min_p)).astype(np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_many_equal_logits_at_a_small_top_k(t):
    """More tokens than a list of candidates holds, all of them equal."""
    import torch
    rng = np.random.default_rng(14)
    z = torch.from_numpy((0.3 * rng.standard_normal((4, 6000))).astype(np.float32)).to(types()[t]).cuda()
    for some in (100, 300, 5000):
        z[:, rng.permutation(6000)[:some]] = 2.0
        for k in (2, 50, 96, 97, 128, 129):
            check(z, [(1.0, 0.9, 0.0, k)], np.array([0.0, 0.3, 0.6, 0.99], np.float32))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_masks_and_rows_without_answer(t):
    import torch
    rng = np.random.default_rng(6)
    low = torch.finfo(types()[t]).min
    cols = 700
    for rule in [(1.0, 1.0, 0.0, 0), (1.0, 0.9, 0.02, 60), (0.7, 0.95, 0.0, 0), (1.0, 1.0, 0.0, 650), (0.0, 1.0, 0.0, 0)]:
        z = torch.from_numpy(rng.standard_normal((10, cols)).astype(np.float32)).to(types()[t]).cuda()
        z[0, 100:] = -math.inf
        z[1] = -math.inf
        z[2] = -math.inf
        z[2, 699] = -3.0
        z[3] = low
        z[4, :690] = low
        z[5, 3] = math.nan
        z[6, 699] = math.inf
        z[7] = math.inf
        z[8, ::2] = -math.inf
        z[9] = torch.finfo(types()[t]).max
        token, _, kept = check(z, [rule], rng.random(10).astype(np.float32))
        assert token[[1, 5, 6, 7]].tolist() == [-1] * 4 and kept[[1, 5, 6, 7]].tolist() == [0] * 4 and token[2] == 699
    bad = [(-1.0, 1.0, 0.0, 0), (math.nan, 1.0, 0.0, 0), (math.inf, 1.0, 0.0, 0), (1.0, math.nan, 0.0, 0), (1.0, 1.0, math.nan, 0)]
    z = torch.zeros((5, 9), dtype=types()[t], device="cuda")
    assert check(z, bad, np.full(5, 0.5, np.float32))[0].tolist() == [-1] * 5


def test_random_numbers_outside_their_range():
    import torch
    z = torch.zeros((6, 300), device="cuda")
    token, _, _ = check(z, [(1.0, 1.0, 0.0, 0)], np.array([-0.5, 1.0, 1.5, math.inf, -math.inf, 0.0], np.float32))
    assert token.tolist() == [0, 299, 299, 299, 0, 0]
    assert draw(z[:1].contiguous(), [(1.0, 1.0, 0.0, 0)], [math.nan])[0].tolist() == [0]


@pytest.mark.parametrize("rule", [(1.0, 1.0, 0.0, 0), (0.8, 0.9, 0.0, 0), (1.0, 1.0, 0.0, 9), (1.2, 0.8, 0.05, 30)])
def test_shares(rule):
    """Over random numbers in equal steps every token comes as often as its share says, but for one."""
    import torch
    rng = np.random.default_rng(8)
    n, cols = 2048, 60
    row = (1.5 * rng.standard_normal(cols)).astype(np.float32)
    z = torch.from_numpy(np.tile(row, (n, 1))).cuda()
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    token, logprob, kept = draw(z, [rule], u)
    assert (np.diff(token) >= 0).all()
    count = np.bincount(token, minlength=cols)
    assert (count > 0).sum() <= kept[0]
    for j in np.unique(token):
        assert abs(count[j] - n * math.exp(logprob[token == j][0])) <= 1 + 1e-3


def test_a_long_row_and_many_rows():
    import torch
    rng = np.random.default_rng(9)
    z = torch.from_numpy((2 * rng.standard_normal((2, 1_000_003))).astype(np.float32)).cuda()
    check(z, [(1.0, 0.9, 0.0, 0), (1.0, 0.99, 0.0, 100000)], np.array([0.37, 0.81], np.float32))
    z = torch.from_numpy((2 * rng.standard_normal((3000, 130))).astype(np.float32)).to(torch.bfloat16).cuda()
    check(z, [(0.9, 0.9, 0.01, 40)], rng.random(3000).astype(np.float32))
    z = torch.zeros((1, K.SAMPLE_COLS_MAX), dtype=torch.bfloat16, device="cuda")
    assert draw(z, [(1.0, 1.0, 0.0, 0)], [0.999])[0][0] == int(float(np.float32(0.999)) * K.SAMPLE_COLS_MAX)


def test_outputs_that_are_not_wanted():
    import torch
    z = torch.randn((4, 100), device="cuda")
    rule, u = [(1.0, 0.9, 0.0, 0)], [0.1, 0.5, 0.7, 0.9]
    whole = draw(z, rule, u)
    for k in range(3):
        part = draw(z, rule, u, outs=tuple(int(j == k) for j in range(3)))
        assert np.array_equal(part[k], whole[k]) and all((part[j] == 77).all() for j in range(3) if j != k)


def test_on_another_stream_and_in_two_graphs():
    import torch
    rng = np.random.default_rng(10)
    z = torch.from_numpy((2 * rng.standard_normal((8, 5000))).astype(np.float32)).to(torch.bfloat16).cuda()
    rules, u = rules_of([(0.9, 0.9, 0.0, 40)]), torch.from_numpy(rng.random(8).astype(np.float32)).cuda()
    import gpu_util as g
    sets = [(torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"),
             workspace(8, 5000)) for _ in range(2)]

    def call(s):
        t, l, k, ws = s
        assert K.lib().karma_k_sample_bf16(g.ptr(z), C.c_uint64(0), g.ptr(rules), 1, g.ptr(u), g.ptr(t), g.ptr(l), g.ptr(k), 8, 5000, g.ptr(ws),
                                           C.c_uint64(ws.numel()), g.stream_ptr()) == 0

    want = draw(z, rules, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(sets[0])
    side.synchronize()
    same = lambda s, w: all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(s, w))
    assert same(sets[0], want)
    graphs = []
    for s in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(s)
        graphs.append(gr)
    for _ in range(4):      # with other numbers and another rule each time, as a server changes them
        u.copy_(torch.rand(8, device="cuda"))
        rules[0, 0] *= 0.9
        want = draw(z, rules, u)
        for s in sets:
            for t in s[:3]:
                t.fill_(5)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(same(s, want) for s in sets)


def test_offsets_beyond_32_bits():
    import torch
    rng = np.random.default_rng(15)
    ld = (1 << 31) + 9
    room = torch.empty(2 * ld + 3000, dtype=torch.bfloat16, device="cuda")
    z = room.as_strided((3, 2000), (ld, 1))
    z.copy_(torch.from_numpy((2 * rng.standard_normal((3, 2000))).astype(np.float32)).to(torch.bfloat16))
    for rules in ([(1.0, 0.9, 0.0, 0)], [(1.0, 1.0, 0.0, 0), (0.8, 0.9, 0.0, 30), (0.0, 1.0, 0.0, 0)]):
        check(z, rules, rng.random(3).astype(np.float32))


def test_two_calls_at_once():
    import torch
    rng = np.random.default_rng(16)
    zs = [torch.from_numpy((2 * rng.standard_normal((300, 9000))).astype(np.float32)).to(t).cuda() for t in (torch.bfloat16, torch.float32)]
    rules, u = rules_of([RULES[r % len(RULES)] for r in range(300)]), torch.from_numpy(rng.random(300).astype(np.float32)).cuda()
    want = [draw(z, rules, u) for z in zs]
    import gpu_util as g
    streams = [torch.cuda.Stream() for _ in zs]
    outs = [(torch.zeros(300, dtype=torch.int32, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, dtype=torch.int32, device="cuda")) for _ in zs]
    torch.cuda.synchronize()
    for _ in range(5):
        for z, s, o, fn in zip(zs, streams, outs, (K.lib().karma_k_sample_bf16, K.lib().karma_k_sample_f32)):
            assert fn(g.ptr(z), C.c_uint64(0), g.ptr(rules), 300, g.ptr(u), *map(g.ptr, o), 300, 9000, None, C.c_uint64(0), C.c_void_p(s.cuda_stream)) == 0
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(np.array_equal(a.cpu().numpy(), b, equal_nan=a.dtype.is_floating_point) for a, b in zip(o, w))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e36, 1.1e37, 1.2e37, 5e37, 1e38, 3e38, 3.4e38])
def test_temperatures_and_logits_up_to_the_largest_number(t, T):
    """Differences of logits that 32 bits do not hold, and that weigh something all the same."""
    import torch
    top = float(torch.finfo(types()[t]).max)
    rules = [(T, 0.95, 0.0, 0), (T, 0.5, 0.0, 0), (T, 1.0, 0.0, 0), (T, 1.0, 0.2, 0), (T, 1.0, 0.0, 3), (T, 0.9, 1e-5, 700), (T, 0.999, 0.0, 700), (T, 1.0, 0.0, 2000)]
    for cols in (2, 5, 900, 4000):
        rng = np.random.default_rng(cols)
        h = rng.uniform(-1, 1, (len(rules), cols)) * top
        h[:, 0], h[:, -1] = top, -top
        few = np.where(h > 0, 3e38, -3e38)      # two values, many of each
        mid = 1e-3 * h
        mid[:, 1::3] = -np.inf
        mid[:, 1] = -top
        for z in (h, few, mid, h / 4 - 0.75 * top):
            z = torch.from_numpy(z).to(types()[t]).cuda()
            for u in (rng.random(len(rules)), np.full(len(rules), 0.9999)):
                check(z, rules, u.astype(np.float32))
