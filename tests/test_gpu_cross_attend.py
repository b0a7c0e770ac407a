"""Attention over an encoder's states on the GPU against 64 bits."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2609_14991_gb300 as tsd  # noqa: E402

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def reference(k, v, lens, q, counts, sources, scale):
    """(out, sum p |v|, the most that a score's terms sum to) in fp64, row by row of the call."""
    outs, mags, tops, at = [], [], [], 0
    heads, dim = q.shape[1:]
    g = heads // k.shape[2]
    for c, s in zip(counts, sources):
        n = k.shape[1] if lens is None else lens[s]
        kk, vv = k[s, :n].double().repeat_interleave(g, 1), v[s, :n].double().repeat_interleave(g, 1)
        x = q[at:at + c].double()
        at += c
        if n == 0 or c == 0:
            outs.append(torch.zeros_like(x)), mags.append(torch.zeros_like(x)), tops.append(torch.zeros(c, heads, 1).to(x))
            continue
        p = torch.softmax(torch.einsum("chd,nhd->chn", x, kk) * scale, -1)
        outs.append(torch.einsum("chn,nhd->chd", p, vv))
        mags.append(torch.einsum("chn,nhd->chd", p, vv.abs()))
        tops.append(torch.einsum("chd,nhd->chn", x.abs(), kk.abs()).amax(-1, keepdim=True) * abs(scale))
    return torch.cat(outs), torch.cat(mags), torch.cat(tops)


def check(got, k, v, lens, q, counts, sources=None, scale=None, fine=False):
    """Bounds: a score is a sum of up to 128 exact products in fp32, eight or sixteen of them at a time
    (2^-22 of the terms' sum each time, truncated: below 2^-18 in all); a weight carries that, its
    exponent's rounding (scores below 2^6: 2^-18) and 2^x's 2^-22, in sum and product both: twice.  Sums over
    the frames in fp32 add below 2^-15 (2^11 steps of 2^-23 and 16 joins, at most).  In the values'
    product a weight is rounded to the states' type, half a step, or (fine) keeps 16 bits.  Then half a step of the result."""
    sources = list(range(len(counts))) if sources is None else sources
    scale = q.shape[2] ** -0.5 if scale is None else scale
    n = sum(counts)
    want, mag, top = reference(k, v, lens, q[:n], counts, sources, scale)
    step = 2.0 ** -16 if fine else torch.finfo(q.dtype).eps / 2
    tol = (step + 2.0 ** -14 + 2 * top * 2.0 ** -18) * mag + torch.finfo(q.dtype).eps / 2 * want.abs() + 2.0 ** -25
    off = (got[:n].double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


def make(n, frames, kv, dim, dtype=BF, seed=0, poison=None, lens=None):
    g = torch.Generator().manual_seed(seed)
    k, v = ((torch.randn(n, frames, kv, dim, generator=g) + 0.3 * torch.randn(kv, dim, generator=g)).to(dtype).cuda() for _ in range(2))
    if poison is not None:
        for i, x in enumerate(lens):
            k[i, x:], v[i, x:] = poison, poison
    return k, v


def queries(rows, heads, dim, dtype=BF, seed=1):
    return (1.5 * torch.randn(rows, heads, dim, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(counts):
    return ints([sum(counts[:i]) for i in range(len(counts) + 1)])


def for_many_rows(n, kv, rows, frames, dim):
    """A call's sizes (rows: tokens * heads of a group) are those of the kernel for many rows per key head."""
    assert frames > 8000 or n * kv * (-(-rows // 16)) * (frames + 330) >= (350e3 if dim == 64 else 200e3)


LENGTHS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 300]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 3, 40, 130])
def test_lengths(dtype, dim, rows):
    """Every end of a step or tile; what lies behind a source's length is NaN."""
    k, v = make(len(LENGTHS), 300, 2, dim, dtype, seed=rows, poison=math.nan, lens=LENGTHS)
    counts = [rows] * len(LENGTHS)
    if rows == 130:
        for_many_rows(len(LENGTHS), 2, 2 * rows, 300, dim)
    q = queries(sum(counts), 4, dim, dtype)
    out = tsd.CrossStates(k, v, ints(LENGTHS)).attend(q, starts=starts_of(counts), max_rows=rows)
    check(out, k, v, LENGTHS, q, counts, fine=rows < 16)
    assert bool((out[:rows] == 0).all())  # no frames


@pytest.mark.parametrize("poison", [math.inf, -math.inf, 6e4])
@pytest.mark.parametrize("rows", [1, 1500])
def test_what_lies_behind(poison, rows):
    lens = [1, 33, 130, 200]
    if rows > 1:
        for_many_rows(4, 1, 2 * rows, 200, 64)
    k, v = make(4, 200, 1, 64, HF, seed=3, poison=poison, lens=lens)
    q = queries(4 * rows, 2, 64, HF)
    out = tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of([rows] * 4), max_rows=rows)
    check(out, k, v, lens, q, [rows] * 4)


@pytest.mark.parametrize("group", [1, 2, 3, 7, 16, 17, 64])
@pytest.mark.parametrize("kv", [1, 3])
@pytest.mark.parametrize("counts", [[1, 1], [5, 0, 2], [1, 33, 9]])
def test_groups_and_ragged_rows(group, kv, counts):
    n, lens = len(counts), [70, 260, 111][:len(counts)]
    k, v = make(n, 260, kv, 64, seed=group, poison=math.nan, lens=lens)
    q = queries(sum(counts), kv * group, 64)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of(counts), max_rows=max(counts)), k, v, lens, q, counts)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 16, 17, 33, 43, 64])
@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 128)])
def test_groups_of_many_rows(group, dtype, dim):
    counts, lens = [600 // group + 1, 0, 300 // group + 1, 1], [400, 399, 131, 0]
    for_many_rows(4, 4, max(counts) * group, 400, dim)
    k, v = make(4, 400, 4, dim, dtype, seed=group, poison=math.nan, lens=lens)
    q = queries(sum(counts), 4 * group, dim, dtype)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of(counts), max_rows=max(counts)), k, v, lens, q, counts)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("counts", [[127], [128], [129], [255], [256], [257], [1, 511, 0, 513], [700, 3]])
def test_row_tiles(dim, counts):
    lens = [1490, 400, 1, 1333][:len(counts)]
    for_many_rows(len(counts), 32, max(counts), 1500, dim)
    k, v = make(len(counts), 1500, 32, dim, seed=sum(counts))
    q = queries(sum(counts), 32, dim)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of(counts), max_rows=max(counts)), k, v, lens, q, counts)


@pytest.mark.parametrize("max_rows", [None, 1, 16, 300, 10 ** 9])
def test_results_do_not_depend_on_the_bound(max_rows):
    """Rows without a bound, with one too low and with one too high."""
    counts, lens = [1, 300, 20, 0, 2], [500, 77, 300, 9, 1]
    for_many_rows(5, 4, 300 * 2, 500, 64)
    k, v = make(5, 500, 4, 64, seed=9)
    q = queries(sum(counts), 8, 64)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of(counts), max_rows=max_rows), k, v, lens, q, counts)


@pytest.mark.parametrize("rows", [1, 100])
@pytest.mark.parametrize("frames", [1, 5000, 40001])
def test_long_sources(rows, frames):
    lens = [frames, max(1, frames // 3)]
    if rows > 1 and frames > 1:
        for_many_rows(2, 1, 4 * rows, frames, 128)
    k, v = make(2, frames, 1, 128, seed=frames)
    q = queries(2 * rows, 4, 128)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of([rows] * 2), max_rows=rows), k, v, lens, q, [rows] * 2)


def test_without_lengths_and_starts():
    k, v = make(3, 50, 2, 64)
    q = queries(3, 2, 64)
    check(tsd.CrossStates(k, v).attend(q), k, v, None, q, [1] * 3, fine=True)
    check(tsd.CrossStates(k, v).attend(q[:2], sources=ints([2, 2])), k, v, None, q, [1] * 2, [2, 2], fine=True)


@pytest.mark.parametrize("rows", [2, 1200])
def test_shared_sources(rows):
    """Sequences over one source, in any order; and their rows as one sequence."""
    if rows > 2:
        for_many_rows(4, 2, rows, 333, 64)
    lens, sources = [40, 333], [1, 0, 1, 1]
    k, v = make(2, 333, 2, 64, seed=2)
    q = queries(4 * rows, 2, 64)
    s = tsd.CrossStates(k, v, ints(lens))
    check(s.attend(q, starts=starts_of([rows] * 4), sources=ints(sources), max_rows=rows), k, v, lens, q, [rows] * 4, sources)
    check(s.attend(q, starts=starts_of([4 * rows]), sources=ints([1]), max_rows=4 * rows), k, v, lens, q, [4 * rows], [1])


@pytest.mark.parametrize("rows", [1, 2500])
@pytest.mark.parametrize("bad", ["source", "negative source", "long", "negative", "rows", "backwards"])
def test_sequences_out_of_range_are_nan(bad, rows):
    if rows > 1:
        for_many_rows(3, 2, rows, 90, 64)
    lens, sources, at = [30, 60, 90], [2, 1, 0], [0, rows, 2 * rows, 3 * rows]
    if bad == "source":
        sources[1] = 3
    elif bad == "negative source":
        sources[1] = -1
    elif bad == "long":
        lens[1] = 91
    elif bad == "negative":
        lens[1] = -1
    elif bad == "rows":
        at[3] = 5 * rows
    else:
        at = [0, rows, 3 * rows, 2 * rows]  # the last sequence's rows end before they begin
    k, v = make(3, 90, 2, 64)
    q = queries(3 * rows, 2, 64)
    out = torch.full_like(q, 7.0)
    tsd.CrossStates(k, v, ints(lens)).attend(q, starts=ints(at), sources=ints(sources), max_rows=rows, out=out)
    nan = [2] if bad == "rows" else [] if bad == "backwards" else [1]
    fine = [0] if bad == "backwards" else [i for i in range(3) if i not in nan]
    for i in nan:
        assert bool(torch.isnan(out[i * rows:(i + 1) * rows]).all())
    for i in fine:
        part = slice(i * rows, (i + 1) * rows)
        check(out[part], k, v, lens, q[part], [rows], [sources[i]])


@pytest.mark.parametrize("counts", [[1, 1], [3, 9000]])
def test_rows_behind_the_last_sequence_stay(counts):
    if sum(counts) > 2:
        for_many_rows(2, 2, sum(counts) // 2, 100, 64)
    k, v = make(2, 100, 2, 64)
    q = queries(sum(counts) + 5, 2, 64)
    out = torch.full_like(q, 7.0)
    tsd.CrossStates(k, v).attend(q, starts=starts_of(counts), out=out)
    check(out, k, v, None, q, counts)
    assert bool((out[sum(counts):] == 7).all())


@pytest.mark.parametrize("rows", [1, 2100])
@pytest.mark.parametrize("dim", [64, 128])
def test_layouts(rows, dim):
    """Keys and values in one projection's rows; heads before frames; frames before sources; shared heads; queries and results likewise."""
    if rows > 1:
        for_many_rows(3, 2, rows, 150, dim)
    n, frames, kv, lens = 3, 150, 2, [150, 20, 99]
    counts = [rows] * n
    qkv = queries(n * rows, 6, dim)
    q = qkv[:, 2:4]
    a, b = make(n, frames, kv, dim, seed=4)
    both = torch.cat([a, b], 2)
    orders = [(both[:, :, :kv], both[:, :, kv:])]
    for order, back in [((0, 2, 1, 3), (0, 2, 1, 3)), ((1, 0, 2, 3), (1, 0, 2, 3)), ((2, 0, 1, 3), (1, 2, 0, 3))]:
        orders.append(tuple(t.permute(order).contiguous().permute(back) for t in (a, b)))
    orders.append(tuple(t[:, :, :1].expand(n, frames, kv, dim) for t in (a, b)))
    orders.append(tuple(t[:1].expand(n, frames, kv, dim) for t in (a, b)))
    orders.append(tuple(t[:, :1].expand(n, frames, kv, dim) for t in (a, b)))
    for k, v in orders:
        out = torch.empty(2, n * rows, dim, dtype=BF, device="cuda").transpose(0, 1)
        tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of(counts), max_rows=rows, out=out)
        check(out, k, v, lens, q, counts)


@pytest.mark.parametrize("rows", [2, 2100])
def test_queries_that_share_memory(rows):
    """One row for all tokens, one head for all heads; odd distances of heads and rows."""
    n, lens = 3, [150, 20, 99]
    k, v = make(n, 150, 2, 64, seed=14)
    s, at = tsd.CrossStates(k, v, ints(lens)), starts_of([rows] * n)
    buf = queries(n * rows, 5, 72)
    for q in (queries(1, 4, 64).expand(n * rows, 4, 64), queries(n * rows, 1, 64).expand(n * rows, 4, 64), buf[:, 1:, 8:]):
        check(s.attend(q, starts=at, max_rows=rows), k, v, lens, q, [rows] * n)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_wide_groups_of_single_rows(dtype):
    """A token per sequence whose group alone is many rows, without starts."""
    n, lens = 64, [(i * 53) % 301 for i in range(64)]
    for_many_rows(n, 4, 64, 300, 64)
    k, v = make(n, 300, 4, 64, dtype, seed=15, poison=math.nan, lens=lens)
    q = queries(n, 256, 64, dtype)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q), k, v, lens, q, [1] * n)


@pytest.mark.parametrize("rows", [1, 4000])
def test_far_sources(rows):
    """Offsets past 2^32 elements."""
    if rows > 1:
        for_many_rows(3, 1, 2 * rows, 70, 64)
    frames, far = 70, 2 ** 31 + 64
    buf = torch.zeros(2 * far + frames * 64, dtype=BF, device="cuda")
    k = buf.as_strided((3, frames, 1, 64), (far, 64, 64, 1))
    a, _ = make(3, frames, 1, 64, seed=6)
    k.copy_(a)
    q = queries(3 * rows, 2, 64)
    check(tsd.CrossStates(k, k).attend(q, starts=starts_of([rows] * 3), max_rows=rows), k, k, None, q, [rows] * 3)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 3.0])
@pytest.mark.parametrize("rows", [2, 3000])
def test_scales(scale, rows):
    if rows > 2:
        for_many_rows(2, 1, 2 * rows, 200, 64)
    k, v = make(2, 200, 1, 64, HF, seed=7)
    q = queries(2 * rows, 2, 64, HF)
    check(tsd.CrossStates(k, v).attend(q, starts=starts_of([rows] * 2), max_rows=rows, scale=scale), k, v, None, q, [rows] * 2, scale=scale)


@pytest.mark.parametrize("rows", [1, 8000])
@pytest.mark.parametrize("rising", [False, True])
def test_maxima_that_move(rows, rising):
    """Scores that rise or fall by hundreds along the frames: each row's maximum follows."""
    if rows > 1:
        for_many_rows(1, 1, rows, 400, 64)
    frames = 400
    k, v = make(1, frames, 1, 64, HF, seed=8)
    ramp = torch.linspace(-200, 200, frames, device="cuda")
    k[0, :, 0, 0] = (ramp if rising else -ramp).half()
    q = queries(rows, 1, 64, HF)
    q[:, :, 0] = 1.0
    q[::3, :, 0] = -1.0
    check(tsd.CrossStates(k, v).attend(q, starts=starts_of([rows]), max_rows=rows, scale=1.0), k, v, None, q, [rows], scale=1.0)


@pytest.mark.parametrize("rows", [1, 1700])
def test_values_at_the_ends(rows):
    """A NaN or infinite key or value reaches the rows of its source and head alone; one frame's result is its values."""
    if rows > 1:
        for_many_rows(4, 2, rows, 100, 64)
    k, v = make(4, 100, 2, 64, HF, seed=5)
    k[0, 99, 0, 3] = math.nan
    v[1, 50, 1, 7] = math.inf
    q = queries(4 * rows, 2, 64, HF)
    out = tsd.CrossStates(k, v, ints([100, 100, 1, 100])).attend(q, starts=starts_of([rows] * 4), max_rows=rows).view(4, rows, 2, 64)
    assert bool(torch.isnan(out[0, :, 0]).all()) and bool(torch.isfinite(out[0, :, 1]).all())
    assert not bool(torch.isfinite(out[1, :, 1, 7]).any()) and bool(torch.isfinite(out[1, :, 0]).all())
    others = [i for i in range(64) if i != 7]
    assert bool(torch.isfinite(out[1, :, 1][:, others]).all())
    assert torch.equal(out[2], v[2, 0].expand(rows, 2, 64))
    assert bool(torch.isfinite(out[3]).all())


@pytest.mark.parametrize("rows", [2, 700])
@pytest.mark.parametrize("hidden", [1, 130, 600])
def test_frames_of_infinite_scores(rows, hidden):
    """Frames whose scores are -inf, the first of a source among them, weigh nothing; where all are, the result is NaN, as the formula's."""
    n, frames, kv = 4, 700, 4
    if rows > 2:
        for_many_rows(n, kv, rows, frames, 64)
    k, v = make(n, frames, kv, 64, HF, seed=hidden)
    q = queries(n * rows, kv, 64, HF)
    q[:, :, 5] = q[:, :, 5].abs() + 0.5
    k[:, :hidden, :, 5] = -math.inf
    k[3, :, 1, 5] = -math.inf
    out = tsd.CrossStates(k, v).attend(q, starts=starts_of([rows] * n), max_rows=rows)
    bad = out.view(n, rows, kv, 64)[3, :, 1]
    assert bool(torch.isnan(bad).all())
    out.view(n, rows, kv, 64)[3, :, 1] = 0
    k[3, hidden:, 1, 5], v[3, hidden:, 1] = 0, 0
    check(out, k[:, hidden:], v[:, hidden:], None, q, [rows] * n)


@pytest.mark.parametrize("rows", [1, 1200])
def test_a_replayed_graph_follows_lengths_and_sources(rows):
    if rows > 1:
        for_many_rows(2, 2, 2 * rows, 300, 64)
    k, v = make(3, 300, 2, 64, seed=11)
    lens, sources = ints([5, 6, 7]), ints([0, 1])
    s = tsd.CrossStates(k, v, lens)
    q, at = queries(2 * rows, 4, 64), starts_of([rows] * 2)
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.attend(q, starts=at, sources=sources, max_rows=rows, out=out)
    for a, b in (([300, 1, 200], [2, 0]), ([0, 299, 128], [1, 1])):
        lens.copy_(ints(a))
        sources.copy_(ints(b))
        q.copy_(queries(2 * rows, 4, 64, seed=a[0]))
        g.replay()
        check(out, k, v, a, q, [rows] * 2, b)
        assert torch.equal(out, s.attend(q, starts=at, sources=sources, max_rows=rows))  # and run to run


@pytest.mark.parametrize("rows", [1, 200])
def test_two_streams_at_once(rows):
    if rows > 1:
        for_many_rows(2, 2, 2 * rows, 3000, 128)
    k, v = make(2, 3000, 2, 128, seed=12)
    s = tsd.CrossStates(k, v)
    q, at = queries(2 * rows, 4, 128), starts_of([rows] * 2)
    want = s.attend(q, starts=at, max_rows=rows)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [s.attend(q, starts=at, max_rows=rows, stream=x) for _ in range(4) for x in (a, b)]
    a.synchronize(), b.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_many_sequences():
    n = 3001
    lens = [(i * 37) % 40 for i in range(n)]
    k, v = make(n, 40, 1, 64, seed=13)
    q = queries(n, 2, 64)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q), k, v, lens, q, [1] * n, fine=True)


@pytest.mark.parametrize("dtype,dim,n", [(BF, 64, 600), (HF, 64, 2000), (BF, 128, 400), (HF, 128, 1300)])
@pytest.mark.parametrize("rows,group", [(1, 1), (3, 5)])
def test_more_units_than_the_device_holds(dtype, dim, n, rows, group):
    lens = [(i * 37) % 301 for i in range(n)]
    k, v = make(n, 300, 1, dim, dtype, seed=n, poison=math.nan, lens=lens)
    q = queries(n * rows, group, dim, dtype)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of([rows] * n), max_rows=rows), k, v, lens, q, [rows] * n, fine=True)


def test_binding_refusals():
    k, v = make(2, 20, 2, 64)
    s = tsd.CrossStates(k, v)
    q, i2 = queries(2, 4, 64), ints([0, 1])
    for kw, word in [(dict(q=q.half()), "q must"), (dict(q=q[0]), "q must"), (dict(q=q[..., :32]), "q must"), (dict(q=q.cpu()), "device"),
                     (dict(q=q[:0]), "rows"), (dict(q=q, sources=i2.long()), "sources"), (dict(q=q, sources=i2.cpu()), "sources"),
                     (dict(q=q, starts=i2.cpu()), "starts"), (dict(q=q, starts=i2[:1]), "n \\+ 1"), (dict(q=q, starts=i2, sources=i2), "n \\+ 1"),
                     (dict(q=q, out=q.float()), "out must"), (dict(q=q, out=q[:1]), "out must"),
                     (dict(q=torch.cat([q, q], 2)[..., ::2]), "adjacent")]:
        with pytest.raises(ValueError, match=word):
            s.attend(**kw)
    for kw, word in [(dict(q=q[:, :3]), "heads=3"), (dict(q=queries(3, 4, 64)), "n=3"), (dict(q=q, scale=math.nan), "scale"),
                     (dict(q=q, sources=i2[:1]), "must be n=1"), (dict(q=q, max_rows=-1), "max_rows"),
                     (dict(q=q, out=q[:1].expand(2, 4, 64)), "overlap")]:
        with pytest.raises(tsd.TsdError, match=word):
            s.attend(**kw)
    big = tsd.CrossStates(*make(4, 700, 4, 64))
    x = queries(2800, 4, 64)
    batch, need = tsd.CrossBatchC(4, None, starts_of([700] * 4).data_ptr(), 2800, 700), ctypes.c_int64()
    for_many_rows(4, 4, 700, 700, 64)
    assert tsd.lib().tsd_cross_attend_workspace(big._pc, batch, 4, ctypes.byref(need)) == 0 and need.value > 0
    for space, size in ((None, need.value), (x.data_ptr(), need.value - 1), (x.data_ptr() + 8, need.value)):  # refused, not written
        assert tsd.lib().tsd_cross_attend(big._pc, batch, 4, x.data_ptr(), 256, 64, 0.1, x.data_ptr(), 256, 64, space, size, None) == tsd.TSD_EINVAL
        assert b"workspace" in tsd.lib().tsd_last_error()
    for args, word in [((k, v, i2.long()), "lens"), ((k, v, i2[:1]), "lens"), ((k, v, i2.cpu()), "one device"), ((k, v.cpu()), "one device"),
                       ((torch.cat([k, k], 3)[..., ::2], v), "adjacent"),
                       ((torch.zeros(2, 20, 2, 68, dtype=BF, device="cuda")[..., :64], v), "multiples of 8"),
                       ((torch.zeros(k.numel() + 4, dtype=BF, device="cuda")[4:].view(k.shape), v), "16-byte")]:
        with pytest.raises(ValueError, match=word):
            tsd.CrossStates(*args)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("frames", [5, 33, 64, 100, 129])
def test_weights_of_many_rows_keep_16_bits(dtype, dim, frames):
    """Few frames whose values have either sign: what a weight loses is not averaged away, and the results are small beside it."""
    n, kv, rows = 4, 4, 1100
    for_many_rows(n, kv, rows, frames, dim)
    lens = [frames, frames - 1, 2, 3]
    k, v = make(n, frames, kv, dim, dtype, seed=frames)
    v = torch.where(torch.arange(frames, device="cuda")[:, None, None] % 2 == 0, v.abs(), -v.abs())
    q = queries(n * rows, kv, dim, dtype, seed=frames)
    out = tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of([rows] * n), max_rows=rows)
    check(out, k, v, lens, q, [rows] * n, fine=True)


@pytest.mark.parametrize("max_rows", [None, 1, 300, 10 ** 9])
def test_the_bound_moves_no_result_by_more_than_last_bits(max_rows):
    """Whichever kernel a bound selects keeps 16 bits of a weight."""
    counts, lens = [1, 300, 20, 0, 2], [500, 77, 300, 9, 1]
    k, v = make(5, 500, 4, 64, seed=19)
    q = queries(sum(counts), 8, 64)
    check(tsd.CrossStates(k, v, ints(lens)).attend(q, starts=starts_of(counts), max_rows=max_rows), k, v, lens, q, counts, fine=True)


@pytest.mark.parametrize("rows", [1, 600])
@pytest.mark.parametrize("gap", [14.0, 17.5, 20.6, 23.0, 25.2])
def test_small_weights_of_fp16_states(rows, gap):
    """Frames far below a row's largest, whose values are 0 (an attention sink): the small weights are the result.  Besides
    check()'s bounds a weight is off by half fp16's smallest step, 2^-25, where the largest is 2^14 at least (many rows: 2^7)."""
    n, kv, frames, every = 40, 4, 1500, 300
    if rows > 1:
        for_many_rows(n, kv, rows, frames, 64)
    g = torch.Generator().manual_seed(int(gap))
    k = torch.zeros(n, frames, kv, 64)
    k[..., 0] = -gap + 0.25 * torch.rand(n, frames, kv, generator=g)
    v = 0.5 + torch.rand(n, frames, kv, 64, generator=g)
    k[:, 7::every], v[:, 7::every] = 0, 0
    k, v = k.half().cuda(), v.half().cuda()
    q = torch.zeros(n * rows, kv, 64, dtype=HF, device="cuda")
    q[..., 0] = 1.0
    out = tsd.CrossStates(k, v).attend(q, starts=starts_of([rows] * n), max_rows=rows, scale=math.log(2)).double()
    want, mag, top = reference(k, v, None, q.view(n, rows, kv, 64)[:, 0], [1] * n, list(range(n)), math.log(2))
    small = frames * 2.0 ** (-39 if rows == 1 else -32) * float(v.max()) / (frames // every)  # (the largest, of which there are as many, divide it)
    tol = (2.0 ** -16 + 2.0 ** -14 + 2 * top * 2.0 ** -18) * mag + 2.0 ** -11 * want.abs() + 2.0 ** -25 + small
    off = (out.view(n, rows, kv, 64) - want[:, None]).abs()
    assert bool((off <= tol[:, None]).all()), float((off / tol[:, None]).max())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [1, 1700])
def test_an_infinite_value_is_infinite_in_the_result(dtype, rows):
    """A visible frame with a value of inf, and one of -inf: the results of that dimension are they, as the formula's."""
    if rows > 1:
        for_many_rows(4, 2, rows, 100, 64)
    k, v = make(4, 100, 2, 64, dtype, seed=5)
    k *= 0.25
    v[0, 3, 0, 9], v[1, 50, 1, 7] = math.inf, -math.inf
    q = queries(4 * rows, 2, 64, dtype)
    out = tsd.CrossStates(k, v).attend(q, starts=starts_of([rows] * 4), max_rows=rows).view(4, rows, 2, 64)
    assert bool((out[0, :, 0, 9] == math.inf).all()) and bool((out[1, :, 1, 7] == -math.inf).all())
    out[0, :, 0, 9], out[1, :, 1, 7] = 0, 0
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype,size", [(HF, 3000.0), (BF, 3000.0), (BF, 1e14)])
@pytest.mark.parametrize("scale", [1.0, -1.0])
@pytest.mark.parametrize("rows", [2, 1500])
def test_scores_of_any_finite_size(dtype, size, scale, rows):
    """Scores up to 6e8 (1e30), of which each row's largest leaves the others nothing: the result is its frame's values."""
    n, kv, frames = 4, 1, 200
    if rows > 2:
        for_many_rows(n, kv, 2 * rows, frames, 64)
    g = torch.Generator().manual_seed(int(rows))
    signs = torch.sign(torch.randn(64, generator=g))
    size_of = torch.stack([torch.randperm(frames, generator=g).float() for _ in range(n)]) / frames
    k = (size * size_of[:, :, None, None] * signs).to(dtype).cuda()
    v = torch.randn(n, frames, kv, 64, generator=g).to(dtype).cuda()
    q = (size * (0.5 + 0.5 * torch.rand(n * rows, 2, 1, generator=g)) * signs).to(dtype).cuda()
    out = tsd.CrossStates(k, v).attend(q, starts=starts_of([rows] * n), max_rows=rows, scale=scale).view(n, rows * 2, 64)
    for i in range(n):
        size_in = k[i, :, 0].double() @ signs.double().cuda() * scale
        assert int((size_in == size_in.max()).sum()) == 1
        assert torch.equal(out[i], v[i, int(size_in.argmax()), 0].expand(2 * rows, 64))


@pytest.mark.parametrize("rows", [2, 700])
@pytest.mark.parametrize("hidden", [1, 130, 600])
def test_very_low_scores_behind_infinite_ones(rows, hidden):
    """Two frames of score -3e30 behind and before others of -inf weigh a half each."""
    n, frames, kv = 4, 700, 4
    if rows > 2:
        for_many_rows(n, kv, rows, frames, 64)
    _, v = make(n, frames, kv, 64, seed=hidden)
    k = torch.zeros_like(v)
    k[..., 5] = -math.inf
    two = [hidden, 699]
    k[:, two, :, 5] = -1e20
    q = torch.zeros(n * rows, kv, 64, dtype=BF, device="cuda")
    q[..., 5] = 3e10
    out = tsd.CrossStates(k, v).attend(q, starts=starts_of([rows] * n), max_rows=rows, scale=1.0).view(n, rows, kv, 64)
    want = v[:, two].double().mean(1)[:, None]
    assert bool(((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * v[:, two].double().abs().amax(1)[:, None]).all())
