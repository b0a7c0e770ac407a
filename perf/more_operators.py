"""The measured calls of an attention decoder's layer around the 8-bit cache:
what such a model (a rescoring decoder, a neural LM) computes between its
matrix products besides the cache's own append and attention.

  rotary  ``Rotary``: positions turned into queries and keys before they go to
          the cache, in one launch; half and interleaved pairs, part of the
          head, frequencies scaled for long contexts
  norm    ``residual_norm``: a block's output normed, gated and added to the
          residual stream, and the next block's norm
  cross   ``CrossStates.attend``: attention over an encoder's states of
          another length, a token per hypothesis or whole transcripts

Both forms take the same tensors; the handles hold the state's own.
"""
import math
import random
import types

import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


# ---------------------------------------------------------------- the cases

def _rotary(name, n, new, past, heads, kv, dim, rot, layout, scaling, dtype, given):
    """n sequences of `new` tokens behind `past`; given: the positions come as a
    tensor, else they are those of a cache's call (lens, starts, slots)."""
    return dict(name=name, kind="rotary", n=n, new=new, past=past, heads=heads, kv=kv, dim=dim, rot=rot, layout=layout,
                scaling=scaling, dtype=dtype, given=given)


def _norm(name, n, d, norm, post, gate, scale, dtype, x_dtype):
    return dict(name=name, kind="norm", n=n, d=d, norm=norm, post=post, gate=gate, scale=scale, dtype=dtype, x_dtype=x_dtype)


def _cross(name, n, rows, frames, heads, kv, dim, dtype):
    """n sources of up to `frames` frames, up to `rows` query rows each."""
    return dict(name=name, kind="cross", n=n, rows=rows, frames=frames, heads=heads, kv=kv, dim=dim, dtype=dtype)


def listed():
    return [
        # one hypothesis, one new token: latency
        _rotary("rotary 1 x 1", 1, 1, 777, 8, 8, 64, 64, "half", "none", "bf16", False),
        # a token for each stream of a full server, contexts stretched far past the trained ones
        _rotary("rotary 256 x 1 ramp", 256, 1, 900_000, 32, 8, 128, 128, "half", "ramp", "bf16", False),
        # ragged prompts of a few hypotheses, interleaved pairs, half of the head
        _rotary("rotary 6 x 4000 part", 6, 4000, 0, 16, 2, 128, 64, "interleaved", "linear", "fp16", True),
        # one new token in a small decoder: latency
        _norm("norm 1 x 512", 1, 512, "layer", "none", "none", 1.0, "bf16", "bf16"),
        # a 1040 ms chunk of 256 streams, 0.6B-shaped: half a feed-forward's output on a 32-bit stream
        _norm("norm 3328 x 1024 half step", 3328, 1024, "layer", "none", "none", 0.5, "bf16", "fp32"),
        # an odd width, a gate per row
        _norm("norm 777 x 1537 gated rows", 777, 1537, "rms", "rms", "rows", 0.7, "fp16", "fp16"),
        # prompts of a wide model: norms on both sides of the block, a gate per channel
        _norm("norm 16384 x 4096 both sides", 16384, 4096, "rms", "rms", "channels", 1.0, "bf16", "bf16"),
        # one hypothesis, one token, half a minute of audio (80 ms frames): latency
        _cross("cross 1 x 1 over 375", 1, 1, 375, 8, 8, 64, "bf16"),
        # a server's beams of eight: one token each over up to two minutes
        _cross("cross 64 x 8 over 1500", 64, 8, 1500, 16, 16, 64, "bf16"),
        # an hour of audio, shared key heads, one token each
        _cross("cross 4 x 1 over 45000", 4, 1, 45000, 32, 8, 128, "fp16"),
        # n-best lists rescored in one pass: eight transcripts of some fifty labels per utterance
        _cross("cross 16 x 400 over 750", 16, 400, 750, 8, 8, 128, "bf16"),
        # long ragged texts over long recordings, shared key heads
        _cross("cross 6 x 1100 over 9000", 6, 1100, 9000, 16, 4, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "norm", "cross", "cross"])
    if kind == "rotary":
        dim = rng.choice([32, 64, 80, 96, 128, 128, 256])
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4])
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        n, new = _log_int(rng, 1, 256), rng.choice([1, rng.randint(2, 40), _log_int(rng, 41, 4000)])
        new = max(1, min(new, 28_000_000 // (n * (heads + kv) * dim)))
        c = _rotary("", n, new, _log_int(rng, 1, 5_000_000), heads, kv, dim, rot, rng.choice(["half", "interleaved"]),
                    rng.choice(["none", "linear", "base", "ramp"]), rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    rng.random() < 0.5)
    elif kind == "norm":
        d = _log_int(rng, 8, 12_000)
        n = _log_int(rng, 1, min(16384, 60_000_000 // d))
        dt = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        c = _norm("", n, d, rng.choice(["rms", "layer"]), rng.choice(["none", "rms", "layer"]),
                  rng.choice(["none", "channels", "rows"]), rng.choice([1.0, 0.5, 0.22]), dt, rng.choice([dt, "fp32"]))
    else:
        kv = rng.choice([1, 2, 4, 8, 16])
        heads, dim = kv * rng.choice([1, 1, 2, 3, 4]), rng.choice([64, 128])
        rows = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 1000)])
        frames = _log_int(rng, 1, 20_000)
        n = _log_int(rng, 1, 64)
        n = max(1, min(n, 200_000_000 // (frames * kv * dim), 40_000_000_000 // (rows * frames * heads * dim)))
        c = _cross("", n, rows, frames, heads, kv, dim, rng.choice(["bf16", "bf16", "fp16"]))
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ragged(case, key, most):
    """Sizes of a case's sequences, the same at every seed."""
    if case["n"] == 1:
        return [most]
    r = random.Random(case["n"] * 7919 + most * 31 + len(key))
    return [max(1, int(most * r.uniform(0.4, 1.0))) for _ in range(case["n"])]


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(counts):
    return torch.cumsum(torch.tensor([0] + list(counts)), 0).to(torch.int32).to(DEV)


FACTOR, ORIGINAL, LOW, HIGH, MAGNITUDE = 8.0, 4096, 1.0, 32.0, 1.1


def _frequencies(case):
    """Radians per position of each pair, fp64."""
    half = case["rot"] // 2
    base, scaling = 10000.0, case["scaling"]
    if scaling == "base" and half > 1:
        base *= FACTOR ** (half / (half - 1))
    f = base ** (-torch.arange(half, dtype=torch.float64) / half)
    if scaling == "linear":
        f = f / FACTOR
    elif scaling == "ramp":
        keep = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * keep + f / FACTOR * (1 - keep)
    return f


def prepare(case, seed):
    g = _rng(seed)
    s = types.SimpleNamespace(kind=case["kind"], case=case)
    {"rotary": _prepare_rotary, "norm": _prepare_norm, "cross": _prepare_cross}[case["kind"]](s, case, g)
    return s


def _prepare_rotary(s, case, g):
    n, heads, kv, dim, dt = case["n"], case["heads"], case["kv"], case["dim"], TYPES[case["dtype"]]
    new, past = _ragged(case, "new", case["new"]), _ragged(case, "past...", case["past"])
    rows = sum(new)
    # queries and keys stand in one projection's rows, values behind them
    qkv = torch.randn((rows, heads + 2 * kv, dim), generator=g, device=DEV).to(dt)
    s.q, s.k = qkv[:, :heads], qkv[:, heads:heads + kv]
    s.starts = _starts(new)
    s.slots = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    s.lens = torch.empty(n, dtype=torch.int32, device=DEV)
    s.lens[s.slots.long()] = _int([p + c for p, c in zip(past, new)])
    s.positions = None
    if case["given"]:
        s.positions = torch.cat([torch.arange(p, p + c) for p, c in zip(past, new)]).to(torch.int32).to(DEV)
    s.magnitude = MAGNITUDE if case["scaling"] == "ramp" else 1.0
    s.freqs = _frequencies(case).to(DEV)
    s.rotary = None
    if own:
        import paper_2609_14991_gb300 as tsd

        how = None if case["scaling"] == "none" else case["scaling"]
        s.rotary = tsd.Rotary(dim, case["rot"], layout=case["layout"], base=10000.0, scaling=how, factor=FACTOR,
                              original=ORIGINAL, low=LOW, high=HIGH, magnitude=s.magnitude)


def _prepare_norm(s, case, g):
    n, d = case["n"], case["d"]
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    # a residual stream: a few wide channels, and a mean
    wide = 1 + 8 * (torch.rand(d, generator=g, device=DEV) < 0.01)
    s.x = (rand(n, d) * 2 * wide + 0.3).to(TYPES[case["x_dtype"]])
    s.y = (rand(n, d) * 0.7 + 0.05).to(TYPES[case["dtype"]])
    weight = lambda: 1 + 0.2 * rand(d)  # noqa: E731
    s.w, s.pw = weight(), weight()
    s.b, s.pb = (0.1 * rand(d) if case[k] == "layer" else None for k in ("norm", "post"))
    s.gate = None
    if case["gate"] != "none":
        shape = (n, d) if case["gate"] == "rows" else (d,)
        s.gate = torch.tanh(rand(*shape)).to(TYPES[case["dtype"]])
    s.eps = 1e-5


def _prepare_cross(s, case, g):
    n, kv, dim, dt = case["n"], case["kv"], case["dim"], TYPES[case["dtype"]]
    frames = case["frames"]
    lens, rows = _ragged(case, "frames", frames), _ragged(case, "rows", case["rows"]) if case["rows"] > 8 else [case["rows"]] * n

    def states():  # each channel with its own mean, each head with its own spread; the padding is not zero
        x = torch.randn((n, frames, kv, dim), generator=g, device=DEV)
        x *= torch.exp2(torch.rand(kv, 1, generator=g, device=DEV) - 0.5)
        return (x + 0.3 * torch.randn((kv, dim), generator=g, device=DEV)).to(dt)

    s.k, s.v = states(), states()
    # a sequence's source: another order than the call's
    s.sources = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    s.lens = torch.empty(n, dtype=torch.int32, device=DEV)
    s.lens[s.sources.long()] = _int(lens)
    s.counts, s.rows, s.max_rows = rows, sum(rows), max(rows)
    s.starts = _starts(rows)
    s.q = (1.5 * torch.randn((s.rows, case["heads"], dim), generator=g, device=DEV)).to(dt)
    s.scale = 1 / math.sqrt(dim)
    s.states = None
    if own:
        import paper_2609_14991_gb300 as tsd

        s.states = tsd.CrossStates(s.k, s.v, s.lens)


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"rotary": _plain_rotary, "norm": _plain_norm, "cross": _plain_cross}[s.kind](s)


def _run_own(s):
    import paper_2609_14991_gb300 as tsd

    c = s.case
    if s.kind == "rotary":
        if s.positions is not None:
            q, k = s.rotary(s.q, s.k, positions=s.positions)
        else:
            q, k = s.rotary(s.q, s.k, lens=s.lens, starts=s.starts, slots=s.slots)
        return {"q": q, "k": k}
    if s.kind == "norm":
        post = c["post"] if c["post"] != "none" else None
        h, r = tsd.residual_norm(s.x, s.y, norm=c["norm"], weight=s.w, bias=s.b, post=post,
                                 post_weight=s.pw if post else None, post_bias=s.pb, gate=s.gate, scale=c["scale"], eps=s.eps)
        return {"h": h, "r": r}
    return s.states.attend(s.q, starts=s.starts, sources=s.sources, scale=s.scale, max_rows=s.max_rows)


def _turned(x, cos, sin, rot, layout):
    y = x.float()
    if layout == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    u, v = a * cos - b * sin, b * cos + a * sin
    t = torch.cat([u, v], -1) if layout == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([t, y[..., rot:]], -1).to(x.dtype)


def _plain_rotary(s):
    c = s.case
    pos = s.positions
    if pos is None:
        rows = torch.arange(len(s.q), device=DEV)
        i = torch.searchsorted(s.starts[1:], rows, right=True)
        pos = s.lens[s.slots.long()[i]] - (s.starts[1:][i] - rows)
    angle = pos.double()[:, None] * s.freqs  # 64 bits: angles of far positions
    cos, sin = (s.magnitude * f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    return {"q": _turned(s.q, cos, sin, c["rot"], c["layout"]), "k": _turned(s.k, cos, sin, c["rot"], c["layout"])}


def _normed(v, kind, w, b, eps):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * w
    return v if b is None else v + b


def _plain_norm(s):
    c = s.case
    y = s.y.float()
    if c["post"] != "none":
        y = _normed(y, c["post"], s.pw, s.pb, s.eps)
    if s.gate is not None:
        y = y * s.gate.float()
    r = s.x.float() + c["scale"] * y
    return {"h": _normed(r, c["norm"], s.w, s.b, s.eps).to(s.y.dtype), "r": r.to(s.x.dtype)}


def _plain_cross(s):
    c = s.case
    n, kv, g, dim = c["n"], c["kv"], c["heads"] // c["kv"], c["dim"]
    src = s.sources.long()
    t = torch.arange(s.max_rows, device=DEV)
    row = (s.starts[:-1, None] + t).clamp(max=s.rows - 1)
    q = s.q[row].float().view(n, s.max_rows, kv, g, dim).permute(0, 2, 3, 1, 4).reshape(n, kv, g * s.max_rows, dim)
    k, v = s.k[src].float(), s.v[src].float()
    att = (q * s.scale) @ k.permute(0, 2, 3, 1)
    seen = torch.arange(c["frames"], device=DEV) < s.lens[src][:, None]
    att.masked_fill_(~seen[:, None, None], -math.inf)
    att -= att.amax(-1, keepdim=True)
    att = att.exp_()
    att /= att.sum(-1, keepdim=True)
    out = (att @ v.transpose(1, 2)).view(n, kv, g, s.max_rows, dim).permute(0, 3, 1, 2, 4).reshape(n, s.max_rows, kv * g, dim)
    r = torch.arange(s.rows, device=DEV)
    i = torch.searchsorted(s.starts[1:], r, right=True)
    return out[i, r - s.starts[i]].to(s.q.dtype)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind == "rotary":
        values = sum(_ragged(case, "new", case["new"])) * (case["heads"] + case["kv"]) * case["dim"]
        rows = sum(_ragged(case, "new", case["new"]))
        return {"bytes": 2 * SIZE[case["dtype"]] * values + (4 * rows if case["given"] else 12 * case["n"]), "flops": 4 * values}
    if kind == "norm":
        n, d, e, x = case["n"], case["d"], SIZE[case["dtype"]], SIZE[case["x_dtype"]]
        gate = {"none": 0, "channels": e * d, "rows": e * n * d}[case["gate"]]
        vectors = sum({"none": 0, "rms": 4, "layer": 8}[case[k]] for k in ("norm", "post")) * d
        return {"bytes": 2 * n * d * (e + x) + gate + vectors, "flops": 12 * n * d}
    n, kv, heads, dim = case["n"], case["kv"], case["heads"], case["dim"]
    lens = _ragged(case, "frames", case["frames"])
    rows = _ragged(case, "rows", case["rows"]) if case["rows"] > 8 else [case["rows"]] * n
    pairs = sum(a * b for a, b in zip(lens, rows))
    return {"bytes": 4 * sum(lens) * kv * dim + 4 * sum(rows) * heads * dim, "flops": 4 * dim * heads * pairs}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "norm": _exact_norm, "cross": _exact_cross}[case["kind"]](s, case)


def _exact_rotary(s, case):
    rot, out = case["rot"], {}
    new, past = _ragged(case, "new", case["new"]), _ragged(case, "past...", case["past"])
    pos = torch.cat([torch.arange(p, p + c, dtype=torch.float64) for p, c in zip(past, new)]).to(DEV)
    # each pair as a complex number, turned by e^(i angle)
    turn = torch.polar(torch.full((len(pos), rot // 2), s.magnitude, dtype=torch.float64, device=DEV), pos[:, None] * s.freqs)
    i = torch.arange(rot // 2, device=DEV)
    first, second = (i, i + rot // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
    for name, x in (("q", s.q), ("k", s.k)):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def _exact_norm(s, case):
    def norm(v, kind, w, b):
        if kind == "none":
            return v
        top = v.mean(1, keepdim=True) if kind == "layer" else 0.0
        power = ((v - top) ** 2).mean(1, keepdim=True)
        z = (v - top) * torch.rsqrt(power + s.eps) * w.double()
        return z + b.double() if b is not None else z

    rows = max(1, (1 << 25) // case["d"])
    hs, rs = [], []
    for a in range(0, case["n"], rows):
        y = norm(s.y[a:a + rows].double(), case["post"], s.pw, s.pb)
        if case["gate"] == "rows":
            y = y * s.gate[a:a + rows].double()
        elif case["gate"] == "channels":
            y = y * s.gate.double()
        r = s.x[a:a + rows].double() + case["scale"] * y
        rs.append(r)
        hs.append(norm(r, case["norm"], s.w, s.b))
    return {"h": torch.cat(hs), "r": torch.cat(rs)}


def _exact_cross(s, case):
    g, at, outs = case["heads"] // case["kv"], 0, []
    lens, sources = s.lens.tolist(), s.sources.tolist()
    for src, c in zip(sources, s.counts):
        out = torch.empty((c, case["heads"], case["dim"]), dtype=torch.float64, device=DEV)
        k, v = s.k[src, :lens[src]].double(), s.v[src, :lens[src]].double()
        for j in range(case["heads"]):
            a = s.q[at:at + c, j].double() @ k[:, j // g].t() / math.sqrt(case["dim"])
            out[:, j] = torch.softmax(a, 1) @ v[:, j // g]
        outs.append(out)
        at += c
    return torch.cat(outs)
