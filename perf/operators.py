"""Operators of a language model's training step beside attention and the fully connected layers: a gated linear recurrence,
log probabilities of given tokens with entropy and top alternatives, and the AdamW step over many tensors.

With `own` a pass calls the library's entry points (`karma_k_gated_scan_*`, `karma_k_token_logprob_*`, `karma_k_adamw`);
without, it computes the same from elementary torch operations.
"""
import ctypes as C
import math

import torch

own = False

MARK = 256          # tokens between the states that the recurrence keeps for its backward pass
BLOCK = 64          # values that share a scale where the optimiser's states have 8 bits


# ---------------------------------------------------------------------------------------- the listed cases
def listed():
    return [
        # Single tokens of 64 sequences, each with the state it left off at: the recurrence of a model that generates.
        dict(name="scan_single_tokens", kind="scan", way="fwd", type="bf16", sequences=64, tokens=64, channels=1024, ragged=False, state=True),
        # Prompts of uneven length, packed one behind the other, gates and inputs side by side as one projection leaves them.
        dict(name="scan_prompts", kind="scan", way="fwd", type="bf16", sequences=13, tokens=6011, channels=4256, ragged=True, state=True),
        # One document of 65536 tokens, forward: the longest.
        dict(name="scan_long", kind="scan", way="fwd", type="bf16", sequences=1, tokens=65536, channels=2048, ragged=False, state=False),
        # The benchmark transformer's batch (32 x 1024 tokens of 1024 channels), backward.
        dict(name="scan_backward", kind="scan", way="bwd", type="bf16", sequences=32, tokens=32768, channels=1024, ragged=False, state=False),
        # Three sequences of an odd length and an odd number of channels in fp32, forward and backward, with states.
        dict(name="scan_odd_f32", kind="scan", way="both", type="f32", sequences=3, tokens=2331, channels=777, ragged=False, state=True),
        # The next token of eight requests: few rows, a vocabulary of 51200, twenty alternatives.
        dict(name="logprob_next_tokens", kind="logprob", way="fwd", type="bf16", rows=8, cols=51200, top=20, masked=0, temperature=0.7),
        # Scoring a chunk of 4096 tokens over the benchmark's vocabulary, with entropy and five alternatives.
        dict(name="logprob_score", kind="logprob", way="fwd", type="bf16", rows=4096, cols=32000, top=5, masked=0, temperature=1.0),
        # The gradient of a loss of log probabilities with an entropy term over the largest workloads' vocabulary.
        dict(name="logprob_gradient", kind="logprob", way="bwd", type="bf16", rows=4096, cols=51200, top=0, masked=0, temperature=1.0),
        # An odd vocabulary in fp32, a part of it not allowed, forward and backward.
        dict(name="logprob_odd_f32", kind="logprob", way="both", type="f32", rows=301, cols=50021, top=8, masked=1000, temperature=1.3),
        # The tests' MLP (8 layers of 256): sixteen small tensors, states in 32 bits.
        dict(name="adamw_mlp", kind="adamw", layout="mlp", width=256, depth=8, bits=32),
        # The 200-layer bottleneck network: over 600 tensors, most of them vectors, states in 32 bits.
        dict(name="adamw_many_tensors", kind="adamw", layout="bottleneck", width=64, depth=66, bits=32),
        # One block of the 17B-parameter transformer, states in 8 bits, which are then read out as values.
        dict(name="adamw_block_8bit", kind="adamw", layout="transformer", width=4256, depth=1, bits=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["scan", "scan", "logprob", "logprob", "adamw"])
    if kind == "scan":
        channels = _log_int(rng, 16, 4352)
        if rng.random() < 0.7:
            channels = (channels + 7) // 8 * 8
        tokens = _log_int(rng, 1, min(65536, (1 << 26) // channels))
        ragged = rng.random() < 0.5
        sequences = _log_int(rng, 1, max(1, min(128, tokens)))
        if not ragged:
            tokens = max(1, tokens // sequences) * sequences
        return dict(kind=kind, way=rng.choice(["fwd", "bwd", "both"]), type=rng.choice(["bf16", "bf16", "f32"]), sequences=sequences,
                    tokens=tokens, channels=channels, ragged=ragged, state=rng.random() < 0.5)
    if kind == "logprob":
        cols = _log_int(rng, 100, 160000)
        if rng.random() < 0.6:
            cols = (cols + 7) // 8 * 8
        rows = _log_int(rng, 1, max(1, min(16384, (1 << 27) // cols)))
        return dict(kind=kind, way=rng.choice(["fwd", "bwd", "both"]), type=rng.choice(["bf16", "bf16", "f32"]), rows=rows, cols=cols,
                    top=rng.choice([0, 1, 5, 20, 50]), masked=rng.choice([0, 0, cols // 3]), temperature=round(rng.uniform(0.5, 1.5), 2))
    layout = rng.choice(["mlp", "bottleneck", "transformer"])
    width = {"mlp": lambda: _log_int(rng, 30, 2000), "bottleneck": lambda: 8 * rng.randint(2, 8),
             "transformer": lambda: 8 * _log_int(rng, 16, 256)}[layout]()
    return dict(kind=kind, layout=layout, width=width, depth=rng.randint(1, 8), bits=rng.choice([32, 8]))


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


def _parameters(case):
    return sum(math.prod(s) for s in _shapes(case))


def work(case):
    if case["kind"] == "scan":
        e, n, c = (2 if case["type"] == "bf16" else 4), case["tokens"], case["channels"]
        moved = {"fwd": 3, "bwd": 5, "both": 6}[case["way"]] * n * c * e
        states = (2 if case["way"] == "fwd" else 3) * case["sequences"] * c * 4 if case["state"] else 0
        return {"bytes": moved + states, "flops": {"fwd": 10, "bwd": 20, "both": 25}[case["way"]] * n * c}
    if case["kind"] == "logprob":
        e, n = (2 if case["type"] == "bf16" else 4), case["rows"] * case["cols"]
        return {"bytes": (1 if case["way"] == "fwd" else 2) * n * e, "flops": {"fwd": 6, "bwd": 8, "both": 14}[case["way"]] * n}
    n = _parameters(case)
    # 8 bits: codes and scales are read and written, and the states then given as values
    return {"bytes": n * (28 if case["bits"] == 32 else 24 + 16 / BLOCK), "flops": (15 if case["bits"] == 32 else 50) * n}


# ------------------------------------------------------------------------------------------------------- inputs
class _Draw:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(mean, std, generator=self.gen).to(dtype)

    def ints(self, shape, lo, hi, dtype=torch.int32):
        return torch.randint(lo, hi, shape, device="cuda", dtype=dtype, generator=self.gen)


TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _prepare_scan(case, seed):
    rnd, t, n, c, s = _Draw(seed), TYPES[case["type"]], case["tokens"], case["channels"], case["sequences"]
    rows = n + (5 if case["ragged"] else 0)         # a packed batch has rows behind its last sequence
    # memories of two to some 150 tokens, by channel
    gate = rnd.normal((rows, c)).add_(torch.linspace(0, 5, c, device="cuda"))
    both = torch.empty((rows, 2 * c), dtype=t, device="cuda")
    both[:, :c], both[:, c:] = gate, rnd.normal((rows, c))
    st = dict(case=case, gate=both[:, :c], x=both[:, c:], h=torch.ones((rows, c), dtype=t, device="cuda"), starts=None, h0=None, h_last=None,
              dh=None, dh_last=None, dh0=None, dgate=None, dx=None, marks=None)
    if case["ragged"]:
        cuts = torch.sort(rnd.ints((s - 1,), 0, n + 1))[0]
        st["starts"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)]).int()
    if case["state"]:
        st["h0"], st["h_last"] = rnd.normal((s, c), 0.5), torch.zeros((s, c), device="cuda")
    st["marks"] = torch.zeros((-(-rows // MARK), c), device="cuda")
    if case["way"] != "fwd":
        st["dh"] = rnd.normal((rows, c), 0.1, dtype=t)
        st["dgate"], st["dx"] = torch.ones((rows, c), dtype=t, device="cuda"), torch.ones((rows, c), dtype=t, device="cuda")
        if case["state"]:
            st["dh_last"], st["dh0"] = rnd.normal((s, c), 0.1), torch.zeros((s, c), device="cuda")
    if case["way"] == "bwd":        # what the forward pass left: the state before every MARK-th token
        h = _plain_states(st)
        seq, first = _places(st)
        before = torch.cat([h.new_zeros(1, c), h[:-1]])[::MARK]
        st["marks"].copy_(torch.where(first[::MARK, None], torch.zeros_like(before), before))
    return st


def _prepare_logprob(case, seed):
    rnd, t, rows, cols = _Draw(seed), TYPES[case["type"]], case["rows"], case["cols"]
    z = rnd.normal((rows, cols), 2.0)
    tokens = rnd.ints((rows,), 0, cols)
    z[torch.arange(rows, device="cuda"), tokens.long()] += 6.0          # the text is likelier than chance
    if case["masked"]:
        z[:, rnd.ints((case["masked"],), 0, cols).long()] = float("-inf")
    tokens[3::17] = -1                                                  # padding
    z = z.to(t)
    f32 = lambda *shape: torch.zeros(shape, dtype=torch.float32, device="cuda")
    st = dict(case=case, logits=z, tokens=tokens, logprob=f32(rows), entropy=f32(rows), stats=f32(rows, 2), top_logprob=f32(rows, case["top"]),
              top_id=torch.zeros((rows, case["top"]), dtype=torch.int32, device="cuda"))
    if case["way"] != "fwd":
        st.update(dlogprob=rnd.normal((rows,), 1.0 / rows, -1.0 / rows), dentropy=rnd.normal((rows,), 0.1 / rows), dlogits=torch.zeros_like(z))
    if case["way"] == "bwd":        # what the forward pass left
        zf = z.float()
        m = zf.amax(1)
        st["stats"] = torch.stack([m, ((zf - m[:, None]) / case["temperature"]).exp().sum(1).log()], 1).contiguous()
        lp = (zf - m[:, None]) / case["temperature"] - st["stats"][:, 1:]
        st["entropy"] = -torch.where(lp > -math.inf, lp.exp() * lp, torch.zeros_like(lp)).sum(1)
    return st


def _prepare_adamw(case, seed):
    rnd, shapes = _Draw(seed), _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    up = lambda n: -(-n // BLOCK) * BLOCK
    total = sum(up(n) for n in sizes)       # one allocation per kind of buffer, each tensor on a boundary of BLOCK values
    st = dict(case=case, sizes=sizes, decay=[0.1 if len(s) > 1 else 0.0 for s in shapes], lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=0.83,
              step=1200, seed=seed & 0xffffffff, w=rnd.normal((total,), 0.02), g=rnd.normal((total,), 1e-3, dtype=torch.bfloat16),
              out=torch.zeros((total,), dtype=torch.bfloat16, device="cuda"))
    if case["bits"] == 32:
        st["m"], st["v"] = rnd.normal((total,), 3e-4), rnd.normal((total,), 1e-3).square_()
    else:
        st["m"], st["v"] = rnd.ints((total,), -127, 128, torch.int8), rnd.ints((total,), 1, 256, torch.uint8)
        st["m_scale"], st["v_scale"] = (rnd.normal((total // BLOCK,), 1.0).abs_().add_(0.5).mul_(k) for k in (8e-6, 6e-11))
    st["at"] = [sum(up(n) for n in sizes[:k]) for k in range(len(sizes))]
    if case["bits"] == 8:
        for a, n in zip(st["at"], sizes):       # nothing behind a tensor in its last block
            st["m"][a + n:a + up(n)], st["v"][a + n:a + up(n)] = 0, 0
        st["m_values"], st["v_values"] = (torch.zeros((total,), dtype=torch.float32, device="cuda") for _ in range(2))
    return st


def prepare(case, seed):
    return {"scan": _prepare_scan, "logprob": _prepare_logprob, "adamw": _prepare_adamw}[case["kind"]](case, seed)


# ------------------------------------------------------------------------------------------------ the plain forms
def _places(st):
    """The sequence of every row, and whether the row is its first; rows behind the last sequence belong to none."""
    rows, s = st["gate"].shape[0], st["case"]["sequences"]
    at = torch.arange(rows, device="cuda", dtype=torch.int32)
    starts = st["starts"] if st["starts"] is not None else torch.arange(s + 1, device="cuda", dtype=torch.int32) * (rows // s)
    seq = torch.searchsorted(starts, at, right=True) - 1
    return seq, (starts[seq.clamp(max=s - 1)] == at) & (seq < s)


def _bounds(st):
    rows, s = st["gate"].shape[0], st["case"]["sequences"]
    starts = st["starts"].long() if st["starts"] is not None else torch.arange(s + 1, device="cuda") * (rows // s)
    return starts[:-1], starts[1:]


def _scan(a, u):
    """y_t = a_t y_{t-1} + u_t over the first dimension, by doubling: after the step of width d, y_t holds 2 d terms.  Both are overwritten."""
    d = 1
    while d < a.shape[0]:
        u[d:] = u[d:] + a[d:] * u[:-d]
        a[d:] = a[d:] * a[:-d]
        d *= 2
    return u


def _plain_states(st):
    f, x = st["gate"].float(), st["x"].float()
    b = 1 / (1 + f.exp())
    seq, first = _places(st)
    begin, end = _bounds(st)
    u = b * x
    if st["h0"] is not None:
        row = begin.clamp(max=f.shape[0] - 1)
        u.index_add_(0, row, torch.where((begin < end)[:, None], (1 - b[row]) * st["h0"], torch.zeros_like(st["h0"])))
    return _scan(torch.where(first[:, None], torch.zeros_like(b), 1 - b), u)


def _plain_scan(st):
    case, begin, end = st["case"], *_bounds(st)
    seq, first = _places(st)
    inside = (seq < case["sequences"])[:, None]
    h, t = _plain_states(st), st["h"].dtype
    out = {}
    filled = (begin < end)[:, None]
    if case["way"] != "bwd":
        out["h"] = torch.where(inside, h.to(t), st["h"])
        if case["state"]:
            out["h_last"] = torch.where(filled, h[(end - 1).clamp(min=0)], st["h0"])
    if case["way"] == "fwd":
        return out
    rows = h.shape[0]
    f, x = st["gate"].float(), st["x"].float()
    b = 1 / (1 + f.exp())
    before = torch.cat([h.new_zeros(1, h.shape[1]), h[:-1]])
    before = torch.where(first[:, None], before.new_zeros(()), before)
    u = torch.where(inside, st["dh"].float(), b.new_zeros(()))
    row = begin.clamp(max=rows - 1)
    if case["state"]:
        before.index_add_(0, row, torch.where(filled, st["h0"], torch.zeros_like(st["h0"])))
        u.index_add_(0, (end - 1).clamp(min=0), torch.where(filled, st["dh_last"], torch.zeros_like(st["dh_last"])))
    # D_t = u_t + a_{t+1} D_{t+1} inside a sequence: the same scan on the reversed rows
    a = torch.where(first[:, None], torch.zeros_like(b), 1 - b)
    a = torch.cat([a[1:], a.new_zeros(1, a.shape[1])])
    D = _scan(a.flip(0), u.flip(0)).flip(0)
    out["dgate"] = torch.where(inside, (D * (before - x) * b * (1 - b)).to(t), st["dgate"])
    out["dx"] = torch.where(inside, (D * b).to(t), st["dx"])
    if case["state"]:
        out["dh0"] = torch.where(filled, ((1 - b) * D)[row], st["dh_last"])
    return out


def _plain_logprob(st):
    case, z, rows = st["case"], st["logits"].float(), st["logits"].shape[0]
    scale = 1.0 / case["temperature"]
    m = z.amax(1, keepdim=True)
    q = (z - m) * scale
    e = q.exp()
    s = e.sum(1, keepdim=True)
    lp = q - s.log()
    p = e / s
    entropy = -torch.where(p > 0, p * lp, p).sum(1)
    named = (st["tokens"] >= 0) & (st["tokens"] < z.shape[1])
    token = torch.where(named, st["tokens"], 0).long()[:, None]
    out = {}
    if case["way"] != "bwd":
        out["entropy"] = entropy
        out["logprob"] = torch.where(named, lp.gather(1, token)[:, 0], lp.new_zeros(()))
        if case["top"]:
            # by value, then by the lower index: both in one whole number
            bits = (z + 0.0).view(torch.int32)
            order = (bits ^ ((bits >> 31) & 0x7fffffff)).long() << 32 | (0x7fffffff - torch.arange(z.shape[1], device="cuda"))
            out["top_id"] = (0x7fffffff - (order.topk(case["top"], 1)[0] & 0xffffffff)).int()
            out["top_logprob"] = lp.gather(1, out["top_id"].long())
    if case["way"] != "fwd":
        dlp, dh = torch.where(named, st["dlogprob"], 0.0)[:, None], st["dentropy"][:, None]
        d = -p * dlp - dh * torch.where(p > 0, p * (lp + entropy[:, None]), p)
        d.scatter_add_(1, token, dlp)
        out["dlogits"] = (d * scale).to(st["logits"].dtype)
    return out


def _mix(i, key):
    """A 32-bit hash of value i under a key: multiplications and shifts modulo 2^32."""
    x = (i + key) & 0xffffffff
    x = ((x ^ (x >> 16)) * 0x45c3a2ad) & 0xffffffff
    x = ((x ^ (x >> 15)) * 0x2d51f9b5) & 0xffffffff
    return x ^ (x >> 16)


def _random_bits(st, k, n):
    key = (st["seed"] * 0x9e3779b1 + (k + 1) * 0x7f4a7c15) & 0xffffffff
    x = _mix(torch.arange(n, device="cuda"), key)
    return ((x & 0xffff).double() + 0.5) / 65536, ((x >> 16).double() + 0.5) / 65536


def _plain_adamw(st):
    b1, b2, lr, eps, gs = (float(C.c_float(st[k]).value) for k in ("beta1", "beta2", "lr", "eps", "grad_scale"))
    c1, k2 = 1 / (1 - b1 ** st["step"]), 1 / math.sqrt(1 - b2 ** st["step"])
    eight = st["case"]["bits"] == 8
    for k, n in enumerate(st["sizes"]):
        at = slice(st["at"][k], st["at"][k] + n)
        w, g = st["w"][at], st["g"][at].float()
        decay = float(C.c_float(st["decay"][k]).value)
        if not eight:
            m, v = st["m"][at], st["v"][at]
            g = g * gs
            m.copy_(b1 * m + (1 - b1) * g)
            v.copy_(b2 * v + (1 - b2) * g * g)
        else:
            # in 64 bits: which of two codes a value gets must not hang on the order of the operations
            block = slice(st["at"][k] // BLOCK, st["at"][k] // BLOCK + -(-n // BLOCK))
            each = lambda s: s.double().repeat_interleave(BLOCK)[:n]
            g = g.double() * gs
            qm, qv = st["m"][at].double(), st["v"][at].double()
            m = b1 * (qm * each(st["m_scale"][block])) + (1 - b1) * g
            v = b2 * (qv * qv * each(st["v_scale"][block])) + (1 - b2) * g * g
            most = lambda t: torch.cat([t.float(), t.new_zeros(-n % BLOCK).float()]).view(-1, BLOCK).amax(1)
            sm, sv = most(m.abs()) * (1 / 127), most(v) * (1 / 65025)
            st["m_scale"][block], st["v_scale"][block] = sm, sv
            u, y = _random_bits(st, k, n)
            per = lambda t, s: torch.where(each(s) > 0, t / each(s), t.new_zeros(()))
            st["m"][at] = (per(m, sm) + u).floor().clamp(-127, 127).to(torch.int8)
            z = per(v, sv)
            q = z.sqrt().floor().clamp(0, 255)
            q = (q + (z - q * q > y * (2 * q + 1))).clamp(max=255)
            st["v"][at] = torch.where(z > 0, q.clamp(min=1), q).to(torch.uint8)
            m, v = m.float(), v.float()
        w.copy_(w - lr * decay * w - lr * (c1 * m / (v.sqrt() * k2 + eps)))
        st["out"][at] = w.to(torch.bfloat16)
    if eight:       # what is held in 8 bits, as the values it stands for
        v = st["v"].float().view(-1, BLOCK)
        st["m_values"].copy_((st["m"].float().view(-1, BLOCK) * st["m_scale"][:, None]).view(-1))
        st["v_values"].copy_((v * v * st["v_scale"][:, None]).view(-1))
    return _adamw_outputs(st)


def _adamw_outputs(st):
    m, v = ("m", "v") if st["case"]["bits"] == 32 else ("m_values", "v_values")
    return {"w": st["w"], "out": st["out"], "m": st[m], "v": st[v]}


# ------------------------------------------------------------------------------------------ the library's kernels
def _p(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


def _check(status):
    if status:
        raise RuntimeError("status %d" % status)


def _workspace(st, nbytes):
    """As a user's program keeps it: allocated for the first call, used by the following ones."""
    if "ws" not in st:
        st["ws"] = torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")
    return _p(st["ws"]), C.c_uint64(st["ws"].numel())


def _own_scan(st):
    import paper_2008_11421_amd as K
    case, c = st["case"], st["case"]["channels"]
    if "shape" not in st:
        st["shape"] = K.ScanShape(tokens=st["gate"].shape[0], channels=c, sequences=case["sequences"], ld_gate=2 * c, ld_x=2 * c)
        _workspace(st, K.gated_scan_ws_bytes(st["shape"]))
    queue, shape, (ws, size) = C.c_void_p(torch.cuda.current_stream().cuda_stream), C.byref(st["shape"]), _workspace(st, 0)
    lib, out = K.lib(), {}
    if case["way"] != "bwd":
        fwd = lib.karma_k_gated_scan_fwd_bf16 if case["type"] == "bf16" else lib.karma_k_gated_scan_fwd_f32
        _check(fwd(_p(st["gate"]), _p(st["x"]), _p(st["h0"]), _p(st["starts"]), _p(st["h"]), _p(st["h_last"]),
                   _p(st["marks"]) if case["way"] == "both" else None, shape, ws, size, queue))
        out["h"] = st["h"]
        if case["state"]:
            out["h_last"] = st["h_last"]
    if case["way"] != "fwd":
        bwd = lib.karma_k_gated_scan_bwd_bf16 if case["type"] == "bf16" else lib.karma_k_gated_scan_bwd_f32
        _check(bwd(_p(st["gate"]), _p(st["x"]), _p(st["h0"]), _p(st["starts"]), _p(st["marks"]), _p(st["dh"]), _p(st["dh_last"]),
                   _p(st["dgate"]), _p(st["dx"]), _p(st["dh0"]), shape, ws, size, queue))
        out["dgate"], out["dx"] = st["dgate"], st["dx"]
        if case["state"]:
            out["dh0"] = st["dh0"]
    return out


def _own_logprob(st):
    import paper_2008_11421_amd as K
    case, lib = st["case"], K.lib()
    rows, cols = st["logits"].shape
    if "ws" not in st:
        _workspace(st, K.token_logprob_ws_bytes(rows, cols, case["top"]))
    queue, (ws, size), scale = C.c_void_p(torch.cuda.current_stream().cuda_stream), _workspace(st, 0), C.c_float(1.0 / case["temperature"])
    ld, out = C.c_uint64(cols), {}
    if case["way"] != "bwd":
        fwd = lib.karma_k_token_logprob_fwd_bf16 if case["type"] == "bf16" else lib.karma_k_token_logprob_fwd_f32
        top = case["top"] > 0
        _check(fwd(_p(st["logits"]), ld, _p(st["tokens"]), _p(st["logprob"]), _p(st["entropy"]), _p(st["stats"]),
                   _p(st["top_logprob"]) if top else None, _p(st["top_id"]) if top else None, rows, cols, case["top"], scale, ws, size, queue))
        out["entropy"], out["logprob"] = st["entropy"], st["logprob"]
        if top:
            out["top_id"], out["top_logprob"] = st["top_id"], st["top_logprob"]
    if case["way"] != "fwd":
        bwd = lib.karma_k_token_logprob_bwd_bf16 if case["type"] == "bf16" else lib.karma_k_token_logprob_bwd_f32
        _check(bwd(_p(st["logits"]), ld, _p(st["tokens"]), _p(st["stats"]), _p(st["entropy"]), _p(st["dlogprob"]), _p(st["dentropy"]),
                   _p(st["dlogits"]), ld, rows, cols, scale, queue))
        out["dlogits"] = st["dlogits"]
    return out


def _own_adamw(st):
    import paper_2008_11421_amd as K
    if "tensors" not in st:
        eight = st["case"]["bits"] == 8
        flags = K.ADAMW_GRAD_BF16 | K.ADAMW_OUT_BF16 | (K.ADAMW_STATES_8BIT if eight else 0)
        at = lambda t, k, per=1: t.data_ptr() + st["at"][k] // per * t.element_size()
        st["tensors"] = (K.AdamwTensor * len(st["sizes"]))(*[
            K.AdamwTensor(w=at(st["w"], k), m=at(st["m"], k), v=at(st["v"], k), m_scale=at(st["m_scale"], k, BLOCK) if eight else None,
                          v_scale=at(st["v_scale"], k, BLOCK) if eight else None, grad=at(st["g"], k), out=at(st["out"], k), n=n,
                          weight_decay=st["decay"][k], flags=flags) for k, n in enumerate(st["sizes"])])
        st["now"] = K.AdamwStep(lr=st["lr"], beta1=st["beta1"], beta2=st["beta2"], eps=st["eps"], grad_scale=st["grad_scale"], seed=st["seed"],
                                step=st["step"])
        if eight:
            values = lambda t: (C.c_void_p * len(st["sizes"]))(*[at(t, k) for k in range(len(st["sizes"]))])
            st["values"] = values(st["m_values"]), values(st["v_values"])
    queue = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    _check(K.lib().karma_k_adamw(st["tensors"], len(st["sizes"]), C.byref(st["now"]), None, queue))
    if st["case"]["bits"] == 8:     # read out, as for a checkpoint
        _check(K.lib().karma_k_adamw_states(st["tensors"], len(st["sizes"]), *st["values"], queue))
    return _adamw_outputs(st)


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"scan": _own_scan, "logprob": _own_logprob, "adamw": _own_adamw}[kind](state)
    return {"scan": _plain_scan, "logprob": _plain_logprob, "adamw": _plain_adamw}[kind](state)


# ------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_scan(st):
    """Token by token, as the recurrence is written, and back."""
    case, s = st["case"], st["case"]["sequences"]
    f, x = st["gate"].double(), st["x"].double()
    rows, c = f.shape
    begin, end = (t.tolist() for t in _bounds(st))
    b = torch.sigmoid(-f)
    keep = torch.sigmoid(f)
    h, last = st["h"].double(), torch.zeros((s, c), dtype=torch.float64, device="cuda")
    before, D = torch.zeros_like(f), torch.zeros_like(f)
    first = torch.zeros((s, c), dtype=torch.float64, device="cuda")
    dgate, dx = torch.ones_like(f), torch.ones_like(f)
    add = b * x
    for j in range(s):
        now = st["h0"][j].double() if case["state"] else last.new_zeros(c)
        for t in range(begin[j], end[j]):
            before[t] = now
            now = torch.addcmul(add[t], keep[t], now)
            h[t] = now
        last[j] = now
    out = {}
    if case["way"] != "bwd":
        out["h"] = h
        if case["state"]:
            out["h_last"] = last
    if case["way"] != "fwd":
        dh = st["dh"].double()
        for j in range(s):
            g = st["dh_last"][j].double() if case["state"] else last.new_zeros(c)
            for t in range(end[j] - 1, begin[j] - 1, -1):
                D[t] = dh[t] + g
                g = keep[t] * D[t]
            first[j] = g
        inside = slice(begin[0], end[-1])
        dgate[inside] = (D * (before - x) * keep * b)[inside]
        dx[inside] = (D * b)[inside]
        out["dgate"], out["dx"] = dgate, dx
        if case["state"]:
            out["dh0"] = first
    return out


def _exact_logprob(st):
    case = st["case"]
    rows, cols = st["logits"].shape
    parts = []
    for r in range(0, rows, 1024):
        z = st["logits"][r:r + 1024].double() / float(C.c_double(case["temperature"]).value)
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        H = torch.special.entr(p).sum(1)
        tok = st["tokens"][r:r + 1024].long()
        hot = torch.nn.functional.one_hot(tok.clamp(min=0), cols).double() * (tok >= 0)[:, None]
        part = {}
        if case["way"] != "bwd":
            part["entropy"] = H
            part["logprob"] = torch.where(hot > 0, lp, 0.0).sum(1)
            if case["top"]:
                best, which = torch.sort(st["logits"][r:r + 1024].double(), dim=1, descending=True, stable=True)
                part["top_id"], part["top_logprob"] = which[:, :case["top"]], lp.gather(1, which[:, :case["top"]])
        if case["way"] != "fwd":
            a, e = st["dlogprob"][r:r + 1024].double()[:, None] * (tok >= 0)[:, None], st["dentropy"][r:r + 1024].double()[:, None]
            part["dlogits"] = (a * (hot - p) - e * torch.where(p > 0, p * (lp + H[:, None]), 0.0)) / case["temperature"]
        parts.append(part)
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}


def _exact_adamw(st):
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).item()
    case, b1, b2 = st["case"], f32(st["beta1"]), f32(st["beta2"])
    w, m, v = st["w"].double(), st["m"].double(), st["v"].double()
    if case["bits"] == 8:
        m = (m.view(-1, BLOCK) * st["m_scale"].double()[:, None]).view(-1)
        v = (v.view(-1, BLOCK).square() * st["v_scale"].double()[:, None]).view(-1)
    live = torch.zeros(w.numel(), dtype=torch.bool, device="cuda")      # gaps between tensors stay as they are
    decay = torch.zeros_like(w)
    rand = torch.zeros(w.numel(), dtype=torch.int64, device="cuda")
    word = 1 << 32
    for k, n in enumerate(st["sizes"]):
        a = st["at"][k]
        live[a:a + n], decay[a:a + n] = True, f32(st["decay"][k])
        if case["bits"] == 8:
            x = torch.remainder(torch.arange(n, device="cuda") + st["seed"] * 0x9e3779b1 % word + (k + 1) * 0x7f4a7c15 % word, word)
            x = torch.bitwise_xor(x, x // 65536) * 0x45c3a2ad % word
            x = torch.bitwise_xor(x, x // 32768) * 0x2d51f9b5 % word
            rand[a:a + n] = torch.bitwise_xor(x, x // 65536)
    g = st["g"].double() * f32(st["grad_scale"])
    m1 = torch.lerp(g, m, b1)
    v1 = torch.lerp(g * g, v, b2)
    t = st["step"]
    w1 = w * (1 - f32(st["lr"]) * decay) - f32(st["lr"]) * (m1 / (1 - b1 ** t)) / ((v1 / (1 - b2 ** t)).sqrt() + f32(st["eps"]))
    if case["bits"] == 8:
        pad = lambda q: torch.where(live, q, 0.0).view(-1, BLOCK)
        sm = (pad(m1).abs().float().amax(1) * (1 / 127)).double()[:, None]
        sv = (pad(v1).float().amax(1) * (1 / 65025)).double()[:, None]
        um, uv = (((rand % 65536).double() + 0.5) / 65536).view(-1, BLOCK), ((rand // 65536).double() + 0.5).view(-1, BLOCK) / 65536
        y = torch.nan_to_num(pad(m1) / sm)
        low = y.floor()
        m1 = ((low + (y - low + um >= 1)).clamp(-127, 127) * sm).view(-1)
        z = torch.nan_to_num(pad(v1) / sv)
        low = z.sqrt().floor().clamp(max=255)
        share = (z - low * low) / ((low + 1) ** 2 - low * low)
        q = (low + (share > uv)).clamp(max=255)
        q = torch.where((z > 0) & (q < 1), 1.0, q)
        v1 = (q * q * sv).view(-1)
    w1 = torch.where(live, w1, w)
    out = torch.where(live, w1, st["out"].double())
    return {"w": w1, "out": out, "m": torch.where(live, m1, m), "v": torch.where(live, v1, v)}


def exact(case, seed):
    return {"scan": _exact_scan, "logprob": _exact_logprob, "adamw": _exact_adamw}[case["kind"]](prepare(case, seed))
