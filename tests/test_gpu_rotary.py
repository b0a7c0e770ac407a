"""Rotary positions on the GPU against the formula with exact angles."""
import math
from decimal import Decimal, getcontext

import pytest

torch = pytest.importorskip("torch")
import paper_2609_14991_gb300 as tsd  # noqa: E402

pytestmark = pytest.mark.gpu
PI2 = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def frequencies(rot, base=10000.0, scaling=None, factor=1.0, original=0.0, low=1.0, high=32.0):
    half, out = rot // 2, []
    if scaling == "base" and half > 1:
        base *= factor ** (half / (half - 1))
    for i in range(half):
        f = base ** (-i / half)
        if scaling == "linear":
            f /= factor
        if scaling == "ramp":
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return out


def angles(positions, freqs):
    """p f mod 2 pi in 64 bits, from exact products."""
    getcontext().prec = 50
    t = [Decimal(f) / PI2 for f in freqs]
    return torch.tensor([[float((p * x) % 1 * PI2) for x in t] for p in positions], dtype=torch.float64)


def turned(x, angle, rot, layout, magnitude):
    """(result, |a| + |b| of each turned element's pair) in fp64."""
    y, size = x.double().cpu().clone(), torch.zeros(x.shape, dtype=torch.float64)
    i = torch.arange(rot // 2)
    first, second = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    a, b = y[..., first].clone(), y[..., second].clone()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    y[..., first], y[..., second] = magnitude * (a * c - b * s), magnitude * (b * c + a * s)
    size[..., first] = size[..., second] = abs(magnitude) * (a.abs() + b.abs())
    return y, size


def check(got, x, pos, rot, layout, magnitude=1.0, **scaling):
    """Bounds: of cosine and sine, 2^-24 for the angle's rounding (at most pi / 4 of it), two units of
    2^-24 by CUDA's bounds for sincospif, one for the magnitude; one for each product and the sum:
    below 8 * 2^-24 (|a| + |b|) in all.  The power's last bits: 2^-50 of the angle.  Then half a step of the type."""
    freqs = frequencies(rot, **scaling)
    want, size = turned(x, angles(pos, freqs), rot, layout, magnitude)
    far = max(abs(p) for p in pos) * max(freqs) * 2.0 ** -50
    tol = (8 * 2.0 ** -24 + far) * size + torch.finfo(x.dtype).eps / 2 * want.abs() + 2.0 ** -25
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    rest = got[..., rot:]
    assert torch.equal(rest, x[..., rot:])


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 64), (128, 128), (80, 80), (96, 32), (256, 256), (2, 2), (3, 2), (37, 18), (66, 66), (1024, 1024), (100, 6)])
def test_given_positions(dtype, layout, dim, rot):
    pos = [0, 1, 2, 17, 4095, 131071, 5_000_001, -3]
    r = tsd.Rotary(dim, rot, layout=layout)
    q, k = rand(len(pos), 5, dim, dtype=dtype), rand(len(pos), 2, dim, dtype=dtype, seed=1)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    oq, ok = r(q, k, positions=p)
    check(oq, q, pos, rot, layout)
    check(ok, k, pos, rot, layout)
    alone = r(q, positions=p)
    assert torch.equal(alone, oq)
    # in place, with the same bits
    q2, k2 = q.clone(), k.clone()
    a, b = r(q2, k2, positions=p, out=(q2, k2))
    assert a is q2 and torch.equal(q2, oq) and torch.equal(k2, ok)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", [(80, 26), (128, 100), (64, 2), (72, 72), (72, 64), (96, 80), (37, 36)])
@pytest.mark.parametrize("heads,kv,rows", [(5, 2, 9), (170, 11, 3), (1, 1, 4000), (700, 1, 1)])
def test_parts_of_heads(dtype, layout, dim, rot, heads, kv, rows):
    """Turned parts that do not end at 16 bytes; heads of a row that several CTAs take; what is not turned, an odd number of times 16 bytes."""
    pos = [(i * 7919) % 100000 for i in range(rows)]
    r = tsd.Rotary(dim, rot, layout=layout)
    q, k = rand(rows, heads, dim, dtype=dtype), rand(rows, kv, dim, dtype=dtype, seed=1)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    oq, ok = r(q, k, positions=p)
    check(oq, q, pos, rot, layout)
    check(ok, k, pos, rot, layout)
    r(q, k, positions=p, out=(q, k))
    assert torch.equal(q, oq) and torch.equal(k, ok)


@pytest.mark.parametrize("pos", [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, 10 ** 9])
def test_farthest_positions(pos):
    r = tsd.Rotary(64, base=500000.0)
    q = rand(1, 3, 64, dtype=torch.float32)
    got = r(q, positions=torch.tensor([pos], dtype=torch.int32, device="cuda"))
    check(got, q, [pos], 64, "half", base=500000.0)


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                dict(scaling="ramp", factor=8.0, original=4096, low=1.0, high=32.0),
                                dict(scaling="ramp", factor=8.0, original=8192, low=1.0, high=4.0, base=500000.0), dict(base=0.25)])
@pytest.mark.parametrize("magnitude", [1.0, 1.2079, -0.5])
def test_scalings(kw, magnitude):
    pos = [0, 3, 77777, 999_999]
    r = tsd.Rotary(128, layout="half", magnitude=magnitude, **kw)
    q = rand(len(pos), 4, 128, dtype=torch.float32)
    check(r(q, positions=torch.tensor(pos, dtype=torch.int32, device="cuda")), q, pos, 128, "half", magnitude, **kw)


def test_turning_back():
    r = tsd.Rotary(64)
    q = rand(9, 2, 64, dtype=torch.float32)
    p = torch.arange(9, dtype=torch.int32, device="cuda") * 1000
    back = r(r(q, positions=p), positions=-p)
    # twice the bound of one call, of pairs no longer than sqrt(2) times the largest element
    assert float((back - q).abs().max()) <= 2 * 9 * 2.0 ** -24 * 2 * float(q.abs().max()) * math.sqrt(2)


@pytest.mark.parametrize("counts", [[1], [1, 1, 1, 1], [0, 3, 0, 70, 1], [300, 2], [0, 0, 5], [1] * 100])
@pytest.mark.parametrize("dim", [64, 36])
def test_positions_of_a_cache(counts, dim):
    n, rows = len(counts), sum(counts)
    g = torch.Generator().manual_seed(rows)
    slots = torch.randperm(n + 2, generator=g)[:n]
    past = torch.randint(0, 5000, (n,), generator=g)
    lens = torch.full((n + 2,), -7, dtype=torch.int32)
    lens[slots] = (past + torch.tensor(counts)).int()
    starts = torch.tensor([0] + list(torch.cumsum(torch.tensor(counts), 0)), dtype=torch.int32)
    pos = [int(past[i]) + t for i, c in enumerate(counts) for t in range(c)]
    r = tsd.Rotary(dim)
    q, k = rand(rows + 3, 3, dim), rand(rows + 3, 2, dim, seed=5)  # three rows behind the last sequence's
    oq, ok = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    r(q, k, lens=lens.cuda(), starts=starts.cuda(), slots=slots.int().cuda(), out=(oq, ok))
    check(oq[:rows], q[:rows], pos, dim, "half")
    check(ok[:rows], k[:rows], pos, dim, "half")
    assert bool((oq[rows:] == 7).all()) and bool((ok[rows:] == 7).all())


def test_one_row_per_sequence():
    r = tsd.Rotary(64)
    lens = torch.tensor([5, 900, 1], dtype=torch.int32, device="cuda")
    q = rand(3, 2, 64)
    check(r(q, lens=lens), q, [4, 899, 0], 64, "half")
    slots = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    check(r(q[:2], lens=lens, slots=slots), q[:2], [0, 4], 64, "half")


@pytest.mark.parametrize("bad", ["slot", "negative slot", "short", "negative", "rows"])
@pytest.mark.parametrize("dim,rot", [(64, 32), (36, 6)])
def test_sequences_out_of_range_are_nan(bad, dim, rot):
    r = tsd.Rotary(dim, rot)
    lens = torch.tensor([50, 60, 70], dtype=torch.int32)
    slots = torch.tensor([0, 1, 2], dtype=torch.int32)
    starts = torch.tensor([0, 2, 5, 6], dtype=torch.int32)
    if bad == "slot":
        slots[1] = 3
    elif bad == "negative slot":
        slots[1] = -1
    elif bad == "short":
        lens[1] = 2
    elif bad == "negative":
        lens[1] = -1
    else:
        starts[3] = 9  # the last sequence's rows end past the call's
    q = rand(6, 2, dim)
    out = r(q, lens=lens.cuda(), starts=starts.cuda(), slots=slots.cuda())
    nan = [5] if bad == "rows" else [2, 3, 4]
    for i in range(6):
        assert bool(torch.isnan(out[i]).all()) == (i in nan), i
    fine = [i for i in range(6) if i not in nan]
    pos = [48, 49, 57, 58, 59, 69]
    check(out[fine], q[fine], [pos[i] for i in fine], rot, "half")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_strided_heads(layout, shift):
    """Queries and keys inside one projection's rows, at any alignment; heads before rows."""
    rows, heads, kv, dim = 21, 4, 2, 64
    buf = rand(rows * (heads + 2 * kv) * dim + 16)
    qkv = buf[shift:shift + rows * (heads + 2 * kv) * dim].view(rows, heads + 2 * kv, dim)
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv]
    pos = list(range(100, 100 + rows))
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    r = tsd.Rotary(dim, layout=layout)
    oq, ok = r(q, k, positions=p)
    check(oq, q, pos, dim, layout)
    check(ok, k, pos, dim, layout)
    head_first = rand(heads, rows, dim, seed=3).transpose(0, 1)
    out = torch.empty(heads, rows, dim, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    r(head_first, positions=p, out=out)
    check(out, head_first, pos, dim, layout)
    before = qkv[:, heads + kv:].clone()
    r(q, k, positions=p, out=(q, k))
    assert torch.equal(q, oq) and torch.equal(k, ok) and torch.equal(qkv[:, heads + kv:], before)


def test_a_replayed_graph_follows_lengths():
    r = tsd.Rotary(64)
    lens = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    q = rand(2, 3, 64)
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r(q, lens=lens, out=out)
    for step in range(3):
        lens += 1000
        g.replay()
        check(out, q, [9 + 1000 * (step + 1), 19 + 1000 * (step + 1)], 64, "half")


def test_another_stream():
    r = tsd.Rotary(64)
    s = torch.cuda.Stream()
    p = torch.tensor([4, 5], dtype=torch.int32, device="cuda")
    q = rand(2, 3, 64)
    torch.cuda.synchronize()
    out = r(q, positions=p, stream=s)
    s.synchronize()
    check(out, q, [4, 5], 64, "half")


def test_many_rows():
    """More rows than CTAs of one each, an odd number of them."""
    rows = 30011
    r = tsd.Rotary(64)
    q = rand(rows, 1, 64)
    p = torch.arange(rows, dtype=torch.int32, device="cuda")
    out = r(q, positions=p)
    pick = [0, 1, 7, 8, 9, 15000, 30003, 30009, 30010]
    check(out[pick], q[pick], pick, 64, "half")
    # ... and every row alone has the same bits
    assert torch.equal(torch.cat([r(q[i:i + 1], positions=p[i:i + 1]) for i in pick]), out[pick])


def test_binding_refusals():
    r = tsd.Rotary(64)
    q, k = rand(4, 2, 64), rand(4, 1, 64)
    p = torch.zeros(4, dtype=torch.int32, device="cuda")
    for kw, word in [(dict(q=q), "positions, or"), (dict(q=q, positions=p, lens=p), "positions, or"), (dict(q=q, positions=p, slots=p), "positions, or"),
                     (dict(q=q, positions=p[:3]), "4 entries"), (dict(q=q, positions=p.long()), "int32"), (dict(q=q, positions=p.cpu()), "device"),
                     (dict(q=q.double(), positions=p), "float32"), (dict(q=q[..., :32], positions=p), "64"), (dict(q=q, k=k.half(), positions=p), "k must"),
                     (dict(q=q, k=k[:3], positions=p), "k must"), (dict(q=q.transpose(1, 2).contiguous().transpose(1, 2), positions=p), "adjacent"),
                     (dict(q=q, lens=p, starts=p[:1]), "n \\+ 1"), (dict(q=q, lens=p, slots=p[:2]), "one row"),
                     (dict(q=q, lens=p, slots=p[:2], starts=p), "n \\+ 1"), (dict(q=q, positions=p, out=k), "result of q"), (dict(q=q.cpu(), positions=p), "device")]:
        with pytest.raises(ValueError, match=word):
            r(**kw)


@pytest.mark.parametrize("dim,rot", [(64, 64), (80, 26)])
def test_far_rows(dim, rot):
    """Rows whose offsets pass 2^32 elements, into rows as far and in place."""
    far, pos = 2 ** 31 + 64, [3, 70000, 11]
    r = tsd.Rotary(dim, rot)
    buf = torch.empty(3 * far, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 2, dim), (far, 128, 1))
    y = buf[1024:].as_strided((3, 2, dim), (far, 128, 1))
    src = rand(3, 2, dim)
    x.copy_(src)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    r(x, positions=p, out=y)
    check(y, src, pos, rot, "half")
    r(x, positions=p, out=x)
    assert torch.equal(x, y)
