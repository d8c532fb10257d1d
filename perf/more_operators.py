"""Operators around the transformer's attention and losses: norms of queries and keys for each head with the rotation by position,
sampling of the next token from given random numbers, and the global norm of many gradients with clipping.

With `own` a pass calls the library's entry points (`karma_k_qk_rotary_*`, `karma_k_sample_*`, `karma_k_grad_norm`,
`karma_k_grad_clip`); without, it computes the same from elementary torch operations.
"""
import ctypes as C
import math

import torch

own = False

ONE = 2.0 ** 40         # a row's weights are whole multiples of 1 / ONE of its largest


# ---------------------------------------------------------------------------------------- the listed cases
def listed():
    return [
        # Single tokens of 64 sequences at places of their own, eight key heads for 32 query heads: a model that generates.
        dict(name="qk_single_tokens", kind="qk", way="fwd", type="bf16", tokens=64, seq=0, heads_q=32, heads_k=8, values=True, d=128, rot=128,
             pairs=False, norm=True),
        # A batch of 8 x 1024 tokens of the widest transformer (28 heads of 152): the projection's thirds become the attention's input.
        dict(name="qk_thirds", kind="qk", way="fwd", type="bf16", tokens=8192, seq=1024, heads_q=28, heads_k=28, values=True, d=152, rot=152,
             pairs=False, norm=True),
        # A training batch of 16 x 1024 tokens with shared key heads, backward.
        dict(name="qk_backward", kind="qk", way="bwd", type="bf16", tokens=16384, seq=1024, heads_q=32, heads_k=8, values=False, d=128, rot=128,
             pairs=False, norm=True),
        # An odd number of tokens and heads in fp32, half of a head's columns turned in neighbouring pairs, forward and backward.
        dict(name="qk_odd_f32", kind="qk", way="both", type="f32", tokens=2331, seq=777, heads_q=7, heads_k=3, values=False, d=72, rot=36,
             pairs=True, norm=True),
        # The next token of eight requests, each with the same usual rule, over the largest workloads' vocabulary.
        dict(name="sample_next_tokens", kind="sample", type="bf16", rows=8, cols=51200, masked=0, temperature=0.7, top_k=50, top_p=0.9, min_p=0.0,
             mixed=False),
        # A batch of 256 requests that bring rules of their own.
        dict(name="sample_requests", kind="sample", type="bf16", rows=256, cols=51200, masked=0, temperature=1.0, top_k=40, top_p=0.9, min_p=0.05,
             mixed=True),
        # 4096 continuations side by side over the benchmark's vocabulary, from the whole of the likeliest 95 %.
        dict(name="sample_rollouts", kind="sample", type="bf16", rows=4096, cols=32000, masked=0, temperature=1.0, top_k=0, top_p=0.95, min_p=0.0,
             mixed=False),
        # An odd vocabulary in fp32, a part of it not allowed, from the unchanged distribution.
        dict(name="sample_odd_f32", kind="sample", type="f32", rows=301, cols=50021, masked=1000, temperature=1.3, top_k=0, top_p=1.0, min_p=0.0,
             mixed=False),
        # The tests' MLP (8 layers of 256) in fp32: the norm of sixteen small tensors and the factor for the update.
        dict(name="norm_mlp", kind="grads", layout="mlp", width=256, depth=8, type="f32", out="", each=False),
        # One block of the 17B-parameter transformer: the norm that the update's factor follows from.
        dict(name="norm_block", kind="grads", layout="transformer", width=4256, depth=1, type="bf16", out="", each=False),
        # The 200-layer bottleneck network's 609 gradients, most of them vectors: norms of each and of all, clipped.
        dict(name="clip_many_tensors", kind="grads", layout="bottleneck", width=64, depth=66, type="bf16", out="bf16", each=True),
        # fp32 sums of an odd width, clipped to bf16 for an exchange.
        dict(name="clip_odd_f32", kind="grads", layout="mlp", width=1777, depth=5, type="f32", out="bf16", each=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["qk", "qk", "sample", "sample", "grads"])
    if kind == "qk":
        d = rng.choice([32, 64, 64, 96, 128, 128, 152, 256, 2 * rng.randint(8, 128)])
        rot = rng.choice([d, d, d, d // 4 * 2, 0, 2 * rng.randint(1, d // 2)])
        heads_q = _log_int(rng, 1, 64)
        heads_k = rng.choice([heads_q, max(1, heads_q // 4), max(1, heads_q // 8), rng.randint(1, heads_q)])
        tokens = _log_int(rng, 1, max(1, min(65536, 30_000_000 // ((heads_q + 2 * heads_k) * d))))
        way = rng.choice(["fwd", "fwd", "bwd", "both"])
        return dict(kind=kind, way=way, type=rng.choice(["bf16", "bf16", "f32"]), tokens=tokens, seq=rng.choice([0, 0, rng.randint(1, tokens)]),
                    heads_q=heads_q, heads_k=heads_k, values=way == "fwd" and rng.random() < 0.5, d=d, rot=rot, pairs=rng.random() < 0.3,
                    norm=rng.random() < 0.8 or rot == 0)
    if kind == "sample":
        cols = _log_int(rng, 100, 160000)
        if rng.random() < 0.6:
            cols = (cols + 7) // 8 * 8
        rows = _log_int(rng, 1, max(1, min(8192, (1 << 26) // cols)))
        return dict(kind=kind, type=rng.choice(["bf16", "bf16", "f32"]), rows=rows, cols=cols, masked=rng.choice([0, 0, cols // 3]),
                    temperature=rng.choice([0.0, 0.6, 1.0, round(rng.uniform(0.3, 2.0), 2)]), top_k=rng.choice([0, 0, 1, 20, 50, rng.randint(1, cols)]),
                    top_p=rng.choice([1.0, 0.9, 0.95, round(rng.uniform(0.05, 1.0), 3)]), min_p=rng.choice([0.0, 0.0, 0.02, 0.1]),
                    mixed=rng.random() < 0.4)
    layout = rng.choice(["mlp", "bottleneck", "transformer"])
    width = {"mlp": lambda: _log_int(rng, 30, 2000), "bottleneck": lambda: 8 * rng.randint(2, 8),
             "transformer": lambda: 8 * _log_int(rng, 16, 256)}[layout]()
    kind_of = rng.choice(["bf16", "f32"])
    depth = min(rng.randint(1, 8), max(1, 4_500_000 // (width * width))) if layout == "transformer" else rng.randint(1, 8)
    return dict(kind=kind, layout=layout, width=width, depth=depth, type=kind_of, out=rng.choice(["", "bf16", kind_of]),
                each=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------- sizes and work
def _shapes(case):
    w, depth = case["width"], case["depth"]
    if case["layout"] == "mlp":
        return [s for _ in range(depth) for s in ((w, w), (w,))]
    if case["layout"] == "transformer":
        return [s for _ in range(depth) for s in ((w,), (w,), (3 * w, w), (3 * w,), (w, w), (w,), (w,), (w,), (4 * w, w), (4 * w,), (w, 4 * w), (w,))]
    out, c_in = [(w, 7, 7, 8), (w,), (w,)], w
    for k, share in enumerate((3, 24, 36, 3)):      # the blocks of the 200-layer network's stages, of 66
        c = w << k
        for b in range(max(1, depth * share // 66)):
            out += [(c, c_in), (c,), (c,), (c, 3, 3, c), (c,), (c,), (4 * c, c), (4 * c,), (4 * c,)]
            out += [(4 * c, c_in), (4 * c,), (4 * c,)] if b == 0 else []
            c_in = 4 * c
    return out


def _size(t):
    return 2 if t == "bf16" else 4


def work(case):
    if case["kind"] == "qk":
        n = case["tokens"] * (case["heads_q"] + case["heads_k"]) * case["d"]
        moved = {"fwd": 2, "bwd": 3 if case["norm"] else 2, "both": 4}[case["way"]] * n * _size(case["type"])
        copied = 2 * case["tokens"] * case["heads_k"] * case["d"] * _size(case["type"]) if case["values"] else 0
        return {"bytes": moved + copied + (0 if case["seq"] else 4 * case["tokens"]), "flops": {"fwd": 7, "bwd": 14, "both": 21}[case["way"]] * n}
    if case["kind"] == "sample":
        n = case["rows"] * case["cols"]
        return {"bytes": n * _size(case["type"]) + case["rows"] * 32, "flops": 4 * n}
    n = sum(math.prod(s) for s in _shapes(case))
    return {"bytes": n * (_size(case["type"]) + (_size(case["out"]) if case["out"] else 0)), "flops": (3 if case["out"] else 2) * n}


# ------------------------------------------------------------------------------------------------------- inputs
class _Draw:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(mean, std, generator=self.gen).to(dtype)

    def uniform(self, shape, lo=0.0, hi=1.0):
        return torch.rand(shape, device="cuda", generator=self.gen) * (hi - lo) + lo

    def ints(self, shape, lo, hi, dtype=torch.int32):
        return torch.randint(lo, hi, shape, device="cuda", dtype=dtype, generator=self.gen)


TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _prepare_qk(case, seed):
    rnd, t, n, d = _Draw(seed), TYPES[case["type"]], case["tokens"], case["d"]
    cols = (case["heads_q"] + case["heads_k"] * (2 if case["values"] else 1)) * d
    st = dict(case=case, positions=None, freq=None)
    # columns of uneven size, as a projection gives them
    st["x"] = (rnd.normal((n, cols)) * torch.exp(rnd.normal((cols,), 0.5))).to(t)
    st["y"] = torch.zeros((n, cols), dtype=t, device="cuda")
    st["gammas"] = [rnd.normal((d,), 0.2, 1.0, dtype=t) for _ in range(2)] if case["norm"] else [None, None]
    if not case["seq"]:
        st["positions"] = rnd.ints((n,), 0, 131072)
    if case["rot"]:
        st["freq"] = 10000.0 ** (-torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda") * 2 / case["rot"])
    if case["way"] != "fwd":
        st["dy"] = rnd.normal((n, cols), 0.1, dtype=t)
        st["dx"] = torch.zeros((n, cols), dtype=t, device="cuda")
        st["dgammas"] = [torch.zeros((d,), device="cuda") for _ in range(2)]
    return st


def _prepare_sample(case, seed):
    rnd, rows, cols = _Draw(seed), case["rows"], case["cols"]
    # a broad rest and a few likely tokens; some rows are surer than others
    z = rnd.normal((rows, cols), 2.0)
    z.scatter_add_(1, rnd.ints((rows, 24), 0, cols, torch.int64), rnd.uniform((rows, 24), 2.0, 9.0))
    z.mul_(rnd.uniform((rows, 1), 0.7, 1.4))
    if case["masked"]:
        z[:, rnd.ints((case["masked"],), 0, cols).long()] = float("-inf")
    k = torch.full((rows if case["mixed"] else 1,), case["top_k"], dtype=torch.int32, device="cuda")
    rules = torch.tensor([[case["temperature"], case["top_p"], case["min_p"], 0.0]], device="cuda").repeat(k.numel(), 1)
    if case["mixed"]:       # of twelve requests one wants the likeliest token, some have no limit of one kind or another
        rules[:, 0] *= rnd.uniform((rows,), 0.6, 1.4)
        at = torch.arange(rows, device="cuda")
        rules[at % 12 == 5, 0] = 0.0
        rules[at % 3 == 1, 1] = 1.0
        rules[at % 4 != 2, 2] = 0.0
        k[at % 2 == 1] = 0
    rules[:, 3] = k.view(torch.float32)
    return dict(case=case, logits=z.to(TYPES[case["type"]]), rules=rules.contiguous(), uniform=rnd.uniform((rows,)),
                token=torch.zeros((rows,), dtype=torch.int32, device="cuda"), kept=torch.zeros((rows,), dtype=torch.int32, device="cuda"),
                logprob=torch.zeros((rows,), device="cuda"))


def _prepare_grads(case, seed):
    rnd, sizes = _Draw(seed), [math.prod(s) for s in _shapes(case)]
    up = lambda n: -(-n // 64) * 64
    total = sum(up(n) for n in sizes)       # one allocation, each tensor on a boundary of 64 values
    st = dict(case=case, sizes=sizes, at=[sum(up(n) for n in sizes[:k]) for k in range(len(sizes))], grad_scale=1.0 / 128)
    st["g"] = rnd.normal((total,), 0.1, dtype=TYPES[case["type"]])
    # a bound of 0.3 to 1.2 times what the norm will be about: most steps are clipped
    st["max_norm"] = st["grad_scale"] * 0.1 * math.sqrt(sum(sizes)) * (0.3 + 0.9 * (seed % 8) / 8)
    st["out"] = torch.zeros((total,), dtype=TYPES[case["out"]], device="cuda") if case["out"] else None
    st["norm"], st["factor"] = torch.zeros((1,), device="cuda"), torch.zeros((1,), device="cuda")
    st["norms"] = torch.zeros((len(sizes),), device="cuda") if case["each"] else None
    return st


def prepare(case, seed):
    return {"qk": _prepare_qk, "sample": _prepare_sample, "grads": _prepare_grads}[case["kind"]](case, seed)


# ------------------------------------------------------------------------------------------------ the plain forms
EPS = 1e-6


def _angles(st):
    """cos and sin of every token's pairs, from angles in 64 bits: a far position has few bits left in 32."""
    case = st["case"]
    at = torch.arange(case["tokens"], device="cuda") % case["seq"] if case["seq"] else st["positions"]
    angle = at.double()[:, None, None] * st["freq"]
    return angle.cos().float(), angle.sin().float()


def _turn(v, case, c, s):
    """The first `rot` columns of v [tokens][heads][d], turned."""
    rot, out = case["rot"], v.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., a], out[..., b] = v[..., a] * c - v[..., b] * s, v[..., b] * c + v[..., a] * s
    return out


def _plain_qk(st):
    case, t = st["case"], st["x"].dtype
    n, d, hq, hk = case["tokens"], case["d"], case["heads_q"], case["heads_k"]
    heads = st["x"].view(n, -1, d)
    c, s = _angles(st) if case["rot"] else (None, None)
    y, dx, dgamma = st["y"].view(n, -1, d), [], []
    for (lo, hi), gamma in zip(((0, hq), (hq, hq + hk)), st["gammas"]):
        x = heads[:, lo:hi].float()
        if case["norm"]:
            r = 1 / ((x * x).mean(-1, keepdim=True) + EPS).sqrt()
            v = x * r * gamma.float()
        else:
            v = x
        if case["way"] != "bwd":
            y[:, lo:hi] = (_turn(v, case, c, s) if case["rot"] else v).to(t)
        if case["way"] != "fwd":
            g = st["dy"].view(n, -1, d)[:, lo:hi].float()
            g = _turn(g, case, c, -s) if case["rot"] else g
            if case["norm"]:
                dgamma.append((g * x * r).double().sum((0, 1)).float())
                g = g * gamma.float()
                g = r * g - x * (r * r * r) * (g * x).mean(-1, keepdim=True)
            dx.append(g.to(t))
    if case["way"] != "bwd" and case["values"]:
        y[:, hq + hk:] = heads[:, hq + hk:]
    out = {} if case["way"] == "bwd" else {"y": st["y"]}
    if case["way"] != "fwd":
        out["dx"] = torch.cat(dx, 1).view(n, -1)
        if case["norm"]:
            out["dgamma_q"], out["dgamma_k"] = dgamma
    return out


def _plain_sample(st):
    z, rows = st["logits"].double(), st["logits"].shape[0]
    rules = st["rules"].expand(rows, 4)
    T, top_p, min_p = (rules[:, j:j + 1].double() for j in range(3))
    k = rules[:, 3:4].contiguous().view(torch.int32)
    greedy = T == 0
    m = z.amax(1, keepdim=True)
    e = (z - m) / torch.where(greedy, 1.0, T)
    w = torch.where(greedy, (e == 0).double(), e.exp()).mul_(ONE).round_().long()       # in 64 bits: which token it is hangs on sums of these
    k = torch.where(greedy, 1, torch.where(k == 0, z.shape[1], k))
    order = torch.sort(z, dim=1, descending=True, stable=True)[1]
    ranked = w.gather(1, order)
    rank = torch.arange(z.shape[1], device="cuda")
    inside = rank < k
    ranked = torch.where(inside, ranked, 0)
    upto = ranked.cumsum(1)
    border = torch.where(top_p >= 1, upto[:, -1:], (top_p * upto[:, -1:].double()).ceil().long())
    stays = (upto - ranked < border) & (ranked.double() >= min_p.clamp(max=1) * ONE) | (rank == 0)
    stays &= ranked > 0
    w = torch.where(torch.zeros_like(stays).scatter_(1, order, stays), w, 0)
    del order, ranked, upto
    upto = w.cumsum(1)
    total = upto[:, -1:]
    target = torch.minimum((st["uniform"][:, None].double() * total.double()).floor().long(), total - 1)
    token = torch.searchsorted(upto, target, right=True)
    logprob = torch.where(greedy, 0.0, e.gather(1, token)) - (total.double() / ONE).log()
    return {"token": token[:, 0].int(), "logprob": logprob[:, 0].float(), "kept": stays.sum(1).int()}


def _f32(v):
    return C.c_float(v).value


def _plain_grads(st):
    case = st["case"]
    each = torch.stack([st["g"][a:a + n].double().square().sum() for a, n in zip(st["at"], st["sizes"])])    # in 64 bits: long sums
    scale, most = _f32(st["grad_scale"]), _f32(st["max_norm"])
    norm = scale * each.sum().sqrt()
    factor = (scale * torch.where(norm <= most, 1.0, most / norm)).float()
    out = {"norm": norm.float()[None], "factor": factor[None]}
    if case["each"]:
        out["norms"] = (scale * each.sqrt()).float()
    if case["out"]:
        for a, n in zip(st["at"], st["sizes"]):
            st["out"][a:a + n] = (st["g"][a:a + n].float() * factor).to(st["out"].dtype)
        out["out"] = st["out"]
    return out


# ------------------------------------------------------------------------------------------ the library's kernels
def _p(t, skip=0):
    return C.c_void_p(t.data_ptr() + skip * t.element_size()) if t is not None else None


def _check(status):
    if status:
        raise RuntimeError("status %d" % status)


def _workspace(st, nbytes):
    """As a user's program keeps it: allocated for the first call, used by the following ones."""
    if "ws" not in st:
        st["ws"] = torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")
    return _p(st["ws"]), C.c_uint64(st["ws"].numel())


def _own_qk(st):
    import paper_2008_11421_amd as K
    case, x = st["case"], st["x"]
    hq, hk, d, ld = case["heads_q"], case["heads_k"], case["d"], x.shape[1]
    if "shape" not in st:
        st["shape"] = K.QkShape(tokens=case["tokens"], seq=case["seq"], heads_q=hq, heads_k=hk, heads_v=hk if case["values"] else 0, d=d,
                                rot=case["rot"], flags=(K.QK_NORM if case["norm"] else 0) | (K.QK_PAIRS if case["pairs"] else 0), eps=EPS,
                                ld_q=ld, ld_k=ld, ld_v=ld, ld_yq=ld, ld_yk=ld, ld_yv=ld, ld_dq=ld, ld_dk=ld, ld_dv=ld)
        _workspace(st, K.qk_rotary_ws_bytes(st["shape"]))
    lib, shape, queue, out = K.lib(), C.byref(st["shape"]), C.c_void_p(torch.cuda.current_stream().cuda_stream), {}
    parts = lambda t: (_p(t), _p(t, hq * d), _p(t, (hq + hk) * d) if case["values"] else None)
    gammas, places = [_p(g) for g in st["gammas"]], (_p(st["positions"]), _p(st["freq"]))
    if case["way"] != "bwd":
        fwd = lib.karma_k_qk_rotary_fwd_bf16 if case["type"] == "bf16" else lib.karma_k_qk_rotary_fwd_f32
        _check(fwd(*parts(x), *gammas, *places, *parts(st["y"]), shape, queue))
        out["y"] = st["y"]
    if case["way"] != "fwd":
        bwd = lib.karma_k_qk_rotary_bwd_bf16 if case["type"] == "bf16" else lib.karma_k_qk_rotary_bwd_f32
        dgammas = [_p(g) if case["norm"] else None for g in st["dgammas"]]
        _check(bwd(*parts(st["dy"]), *parts(x)[:2], *gammas, *places, *parts(st["dx"]), *dgammas, shape, *_workspace(st, 0), queue))
        out["dx"] = st["dx"]
        if case["norm"]:
            out["dgamma_q"], out["dgamma_k"] = st["dgammas"]
    return out


def _own_sample(st):
    import paper_2008_11421_amd as K
    rows, cols = st["logits"].shape
    if "ws" not in st:
        _workspace(st, K.sample_ws_bytes(rows, cols))
    fn = K.lib().karma_k_sample_bf16 if st["case"]["type"] == "bf16" else K.lib().karma_k_sample_f32
    _check(fn(_p(st["logits"]), C.c_uint64(cols), _p(st["rules"]), st["rules"].shape[0], _p(st["uniform"]), _p(st["token"]), _p(st["logprob"]),
              _p(st["kept"]), rows, cols, *_workspace(st, 0), C.c_void_p(torch.cuda.current_stream().cuda_stream)))
    return {"token": st["token"], "logprob": st["logprob"], "kept": st["kept"]}


def _own_grads(st):
    import paper_2008_11421_amd as K
    case, n = st["case"], len(st["sizes"])
    if "tensors" not in st:
        flags = (K.GRAD_BF16 if case["type"] == "bf16" else 0) | (K.GRAD_OUT_BF16 if case["out"] == "bf16" else 0)
        at = lambda t, k: t.data_ptr() + st["at"][k] * t.element_size() if t is not None else None
        st["tensors"] = (K.GradTensor * n)(*[K.GradTensor(grad=at(st["g"], k), out=at(st["out"], k), n=st["sizes"][k], flags=flags) for k in range(n)])
        _workspace(st, K.grad_norm_ws_bytes(st["tensors"]))
    lib, queue = K.lib(), C.c_void_p(torch.cuda.current_stream().cuda_stream)
    _check(lib.karma_k_grad_norm(st["tensors"], n, C.c_float(st["max_norm"]), C.c_float(st["grad_scale"]), _p(st["norm"]), _p(st["norms"]),
                                 _p(st["factor"]), *_workspace(st, 0), queue))
    out = {"norm": st["norm"], "factor": st["factor"]}
    if case["each"]:
        out["norms"] = st["norms"]
    if case["out"]:
        _check(lib.karma_k_grad_clip(st["tensors"], n, _p(st["factor"]), queue))
        out["out"] = st["out"]
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"qk": _own_qk, "sample": _own_sample, "grads": _own_grads}[kind](state)
    return {"qk": _plain_qk, "sample": _plain_sample, "grads": _plain_grads}[kind](state)


# ------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_qk(st):
    """Each pair as a complex number, multiplied by e^(i angle); gradients by its conjugate and by the norm's Jacobian."""
    case = st["case"]
    n, d, hq, hk, rot = case["tokens"], case["d"], case["heads_q"], case["heads_k"], case["rot"]
    places = torch.arange(n, device="cuda").remainder(case["seq"]) if case["seq"] else st["positions"]
    turn = None
    if rot:
        angle = torch.outer(places.double(), st["freq"])
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotate(v, by):
        if not rot:
            return v
        head, rest = v[..., :rot], v[..., rot:]
        if case["pairs"]:
            r = torch.view_as_real(torch.view_as_complex(head.reshape(*head.shape[:2], rot // 2, 2).contiguous()) * by).flatten(-2)
        else:
            z = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * by
            r = torch.cat([z.real, z.imag], -1)
        return torch.cat([r, rest], -1)

    x = st["x"].double().view(n, -1, d)
    ys, dxs, dgs = [], [], []
    for k, (x6, gamma) in enumerate(zip(x[:, :hq + hk].split([hq, hk], 1), st["gammas"])):
        gamma = gamma.double() if gamma is not None else 1.0
        size = (x6.square().mean(-1, keepdim=True) + EPS).sqrt() if case["norm"] else 1.0
        unit = x6 / size
        if case["way"] != "bwd":
            ys.append(rotate(unit * gamma, turn))
        if case["way"] != "fwd":
            g = rotate(st["dy"].double().view(n, -1, d)[:, :hq + hk].split([hq, hk], 1)[k], turn.conj() if rot else None)
            dgs.append((g * unit).sum((0, 1)))
            g = g * gamma
            dxs.append((g - unit * (g * unit).mean(-1, keepdim=True)) / size if case["norm"] else g)
    out = {}
    if case["way"] != "bwd":
        out["y"] = torch.cat(ys + [x[:, hq + hk:]], 1).view(n, -1)
    if case["way"] != "fwd":
        out["dx"] = torch.cat(dxs, 1).view(n, -1)
        if case["norm"]:
            out["dgamma_q"], out["dgamma_k"] = dgs
    return out


def _exact_sample(st):
    """Row by row over places in the order of falling logits, found by one sort of whole numbers that hold logit and index."""
    tokens, logprobs, kepts = [], [], []
    rows, cols = st["logits"].shape
    rules = st["rules"].cpu().expand(rows, 4).contiguous()
    limits = rules[:, 3].contiguous().view(torch.int32).tolist()
    values = rules.double().tolist()
    u = st["uniform"].double().tolist()
    at = torch.arange(cols, device="cuda")
    for r in range(rows):
        z32 = st["logits"][r].float() + 0.0
        bits = z32.view(torch.int32).long()
        key = torch.where(bits < 0, -2147483648 - bits, bits) * (1 << 32) + (cols - at)
        order = key.argsort(descending=True)
        z = z32.double()[order]
        T, top_p, min_p, k = values[r][0], values[r][1], min(values[r][2], 1.0), limits[r] or cols
        if T == 0:
            k, T = 1, 1.0
        share = torch.exp((z - z[0]) / T)
        w = torch.round(share * ONE).long()
        w[k:] = 0
        sums = torch.cumsum(w, 0)
        if top_p < 1:
            need = math.ceil(top_p * float(sums[-1].item()))
            w[int((sums < need).sum().item()) + 1:] = 0
        low = w.double() < min_p * ONE
        low[0] = False
        w[low] = 0
        plain = torch.zeros_like(w).index_put_((order,), w)
        sums = plain.cumsum(0)
        total = int(sums[-1].item())
        target = min(int(u[r] * float(total)), total - 1)
        token = (sums <= target).sum()
        tokens.append(token)
        logprobs.append((z32.double()[token] - z[0]) / T - math.log(total / ONE))
        kepts.append((w > 0).sum())
    return {"token": torch.stack(tokens).int(), "logprob": torch.stack(logprobs), "kept": torch.stack(kepts).int()}


def _exact_grads(st):
    case, scale, most = st["case"], _f32(st["grad_scale"]), _f32(st["max_norm"])
    parts = [st["g"][a:a + n].double() for a, n in zip(st["at"], st["sizes"])]
    norms = [float(torch.dot(p, p)) ** 0.5 * scale for p in parts]
    norm = math.sqrt(math.fsum(v * v for v in norms))
    factor = scale * min(1.0, most / norm)
    as_tensor = lambda v: torch.tensor(v, dtype=torch.float64, device="cuda")
    out = {"norm": as_tensor([norm]), "factor": as_tensor([factor])}
    if case["each"]:
        out["norms"] = as_tensor(norms)
    if case["out"]:
        whole = st["out"].double()
        for p, a in zip(parts, st["at"]):
            whole[a:a + p.numel()] = p * factor
        out["out"] = whole
    return out


def exact(case, seed):
    return {"qk": _exact_qk, "sample": _exact_sample, "grads": _exact_grads}[case["kind"]](prepare(case, seed))
