"""The 8-bit paged cache and attention over it against a plain 64-bit model:
what the cache holds bit for bit, whatever the calls' splits; attention at
lengths from one token on, head layouts, windows, sinks and strides; blocks,
slots and lengths out of range; and the calls that a program makes of them."""
import math

import pytest
import torch

import paper_2609_14991_gb300 as tsd
from tests.kv8_util import Batch

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- what the cache holds

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("block,dim", [(16, 64), (32, 64), (64, 64), (16, 128), (32, 128), (64, 128)])
def test_append_holds_the_rounded_tokens(block, dim, dtype):
    b = Batch(tsd, [1, block - 1, block, block + 1, 3 * block + 5, 0], 3, block, dim, dtype, seed=block + dim)
    b.append([1, block - 1, block, block + 1, 3 * block + 5, 0])
    b.check_held()


@pytest.mark.parametrize("rows", [[3000] + [1] * 40, [1] * 50, [0] * 30 + [700]])
def test_append_without_bounds(rows):
    """A prompt among single tokens, and single tokens with and without starts, no bound given."""
    b = Batch(tsd, [x + 20 for x in rows], 1, 16, 64, seed=len(rows), spare_slots=0)
    b.append([17] * len(rows))
    b.append(rows)
    b.check_held()
    if max(rows) == 1:
        k, a = b.rows(len(rows), 1), b.args(rows)
        a["lens"] += 1
        b.cache.append(k, k, a["table"], a["lens"], slots=a["slots"])
        for i, s in enumerate(b.slots):
            b.len[i] += 1
            b.model.append(s, k[i:i + 1], k[i:i + 1])
        b.check_held()


@pytest.mark.parametrize("block", [16, 64])
def test_append_does_not_depend_on_the_splits(block):
    lens = [2 * block + 7, 5, block, 150]
    whole, parts = (Batch(tsd, lens, 2, block, 64, seed=1) for _ in range(2))
    k, v = whole.append(lens)
    at = [sum(lens[:i]) for i in range(4)]
    left = list(lens)
    step = 0
    while sum(left):
        counts = [min(x, (1, 3, block + 1, 2)[(i + step) % 4]) for i, x in enumerate(left)]
        take = lambda t: torch.cat([t[at[i] + lens[i] - left[i]:][:c] for i, c in enumerate(counts)])  # noqa: E731
        parts.append(counts, k=take(k), v=take(v), max_new=max(counts) if step % 2 else None)
        left = [x - c for x, c in zip(left, counts)]
        step += 1
    for name in ("k", "v", "k_scale", "v_scale"):
        x, y = getattr(whole.cache, name), getattr(parts.cache, name)
        for i, s in enumerate(whole.slots):
            for j in range(-(-lens[i] // block)):
                ids = int(whole.table[s, j]), int(parts.table[parts.slots[i], j])
                n = min(block, lens[i] - j * block)
                p, q = x[ids[0]], y[ids[1]]
                assert torch.equal(p[:, :n] if p.dim() == 3 else p, q[:, :n] if q.dim() == 3 else q), (name, i, j)
    parts.check_held()


def test_scales_and_roundings():
    """Zeros, tiny and huge values, subnormals, exact halves, one large value among small ones."""
    b = Batch(tsd, [16] * 7, 1, 16, 64, torch.bfloat16, seed=3)
    k = torch.zeros(7 * 16, 1, 64)
    k[16:32] = 1e-20
    k[32:48] = 2.0 ** 59
    k[48:64] = 1e-39  # a subnormal
    k[64:80] = torch.arange(16 * 64).view(16, 1, 64) % 255 - 127.0  # scale 1: integers
    k[80:96] = (torch.arange(16 * 64).view(16, 1, 64) % 200) / 2 - 40
    k[80, 0, 0] = 127.0  # scale 1: exact halves
    k[96:112] = torch.randn(16, 1, 64, generator=b.g) * 0.01
    k[100, 0, 5] = 50.0
    k = k.to(torch.bfloat16).cuda()
    b.append([16] * 7, k=k, v=k.flip(0).contiguous())
    b.check_held()


def test_quotients_next_to_halves():
    """fp16 values whose quotients by the scale lie as near to halves as they come."""
    b = Batch(tsd, [64], 2, 64, 128, torch.float16, seed=4)
    g = torch.Generator().manual_seed(9)
    top = torch.tensor(1.3701171875)
    s = top * torch.tensor(1 / 127, dtype=torch.float32)
    k = ((torch.randint(-126, 127, (64, 2, 128), generator=g) + 0.5) * s).half()
    k[0, :, 0] = top.half()
    b.append([64], k=k.cuda(), v=k.flip(2).contiguous().cuda())
    b.check_held()


def test_non_finite_tokens_spoil_their_block_and_head_only():
    b = Batch(tsd, [48, 40], 2, 16, 64, seed=5)
    k = b.rows(88, 2)
    v = b.rows(88, 2)
    k[20, 0, 3] = math.nan
    v[50, 1, 0] = math.inf
    v[2, 0, 1] = -2.0 ** 61
    b.append([48, 40], k=k, v=v)
    b.check_held()
    assert bool(torch.isnan(b.cache.k_scale).sum() == 1) and bool(torch.isnan(b.cache.v_scale).sum() == 2)


def test_strided_rows():
    """Keys, values and queries as slices of one projection's output; results into a slice."""
    b = Batch(tsd, [70, 33], 2, 32, 64, seed=6)
    qkv = b.rows(103, 8)  # 4 query heads, 2 key heads, 2 value heads
    b.append([70, 33], k=qkv[:, 4:6], v=qkv[:, 6:8])
    b.check_held()
    out = torch.full((103, 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    b.check_attend([70, 33], 4, q=qkv[:, :4], out=out[:, 1:5])
    assert bool((out[:, 0] == 7).all()) and bool((out[:, 5] == 7).all())
    by_head = b.rows(4 * 103, 1).view(4, 103, 64).transpose(0, 1)  # heads outermost
    b.check_attend([70, 33], 4, q=by_head)


def test_appending_again_from_an_earlier_length():
    """Tokens taken back (up to a block of them) and others appended in their place."""
    for take in (1, 15, 16):
        b = Batch(tsd, [60], 1, 16, 64, seed=7)
        b.append([35])
        b.append([take])
        b.len[0] -= take
        s = b.slots[0]
        b.model.k[s], b.model.v[s] = b.model.k[s][:35], b.model.v[s][:35]
        b.append([20])
        b.check_held()


def test_taking_back_again_and_again():
    """Within the last two blocks reached, to multiples of the block further back, and on from there."""
    b = Batch(tsd, [90], 1, 16, 64, seed=8)
    s = b.slots[0]
    b.append([50])  # block 3
    for to, new in ((40, 3), (33, 1), (34, 13), (45, 30), (64, 2), (50, 9), (32, 1), (33, 20), (16, 5), (21, 30), (0, 3), (2, 40)):
        b.len[0] = to
        b.model.k[s], b.model.v[s] = b.model.k[s][:to], b.model.v[s][:to]
        b.append([new])
        b.check_held()


def test_reads_a_part_and_leaves_rows_behind():
    b = Batch(tsd, [90, 20, 0], 2, 16, 128, seed=8)
    b.append([90, 20, 0])
    b.check_held(tail=33)
    a = b.args([5, 0, 0])
    out = tuple(torch.full((9, 2, 128), 7.0, device="cuda") for _ in range(2))
    b.cache.read(rows=9, out=out, **a)
    assert bool((out[0][5:] == 7).all()) and bool((out[0][:5] != 7).any())


# ---------------------------------------------------------------- attention

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,block", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64)])
@pytest.mark.parametrize("heads,kv", [(2, 2), (6, 2), (16, 1)])
def test_single_tokens(heads, kv, dim, block, dtype):
    lens = [1, 2, 15, 16, 17, 65, 130, 300]
    b = Batch(tsd, lens, kv, block, dim, dtype, seed=heads + dim)
    b.append(lens)
    b.check_attend([1] * len(lens), heads)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (8, 2), (20, 1), (33, 1), (64, 1)])
@pytest.mark.parametrize("counts", [[1, 2, 3], [5, 0, 13], [16, 17, 1], [40, 1, 33]])
def test_chunks(counts, heads, kv):
    """Row tiles of 16, 32 and 64 rows, several of them, and sequences without a row."""
    past = [30, 100, 7]
    b = Batch(tsd, [p + c for p, c in zip(past, counts)], kv, 16, 64, seed=heads)
    b.append(past)
    b.append(counts)
    b.check_attend(counts, heads)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (16, 0), (17, 3), (40, 16), (40, 17), (64, 1), (100, 500), (1000, 4)])
@pytest.mark.parametrize("counts", [[1, 1, 1], [13, 3, 30]])
def test_windows_and_sinks(window, sinks, counts):
    past = [200, 5, 91]
    b = Batch(tsd, [p + c for p, c in zip(past, counts)], 2, 16, 64, seed=window)
    b.append(past)
    b.append(counts)
    b.check_attend(counts, 4, window=window, sinks=sinks)


def test_prompts():
    for block, dim, heads, kv, window in ((16, 64, 2, 2, 0), (64, 128, 4, 2, 0), (32, 128, 3, 1, 77), (64, 64, 8, 1, 0)):
        counts, past = [150, 257, 64], [0, 70, 3]
        b = Batch(tsd, [p + c for p, c in zip(past, counts)], kv, block, dim, seed=dim)
        b.append(past)
        b.append(counts)
        b.check_attend(counts, heads, window=window, sinks=5 if window else 0)


@pytest.mark.parametrize("dim,dtype", [(64, torch.bfloat16), (128, torch.float16)])
@pytest.mark.parametrize("heads,kv,counts,past,window,sinks", [
    (1, 1, [100, 128, 129], [0, 1, 15], 0, 0),        # one row tile, whole and not
    (1, 1, [256, 257, 385], [16, 0, 100], 0, 0),      # two, and the first of the next pair
    (3, 1, [97, 171, 0], [300, 5, 40], 0, 0),         # a group that does not divide a tile
    (4, 2, [200, 33, 130], [0, 700, 64], 0, 0),
    (2, 1, [300, 64, 150], [20, 400, 129], 50, 0),    # windows inside a tile, across tiles, with sinks
    (2, 2, [150, 260, 128], [200, 333, 1000], 200, 4),
    (8, 1, [40, 13, 100], [600, 20, 0], 17, 33),
    (64, 1, [7, 2, 9], [1000, 0, 90], 0, 0),
])
def test_row_tiles(heads, kv, counts, past, window, sinks, dim, dtype):
    """Prompts in tiles of 128 rows and 128 keys; also with hints that split their keys over CTAs, and
    hints too small, so that a CTA takes several row tiles."""
    b = Batch(tsd, [p + c for p, c in zip(past, counts)], kv, 16 if window else 64, dim, dtype, seed=heads + dim)
    b.append(past)
    b.append(counts)
    b.check_held()
    for kw in (dict(max_new=max(counts)), dict(max_new=96, max_len=64)):
        b.check_attend(counts, heads, window=window, sinks=sinks, **kw)


@pytest.mark.parametrize("past", [9, 10, 16])
def test_row_tiles_with_empty_shares_of_keys(past):
    """More shares than a row tile has key tiles, its units 1 more than whole key tiles; a CTA takes several row tiles."""
    b = Batch(tsd, [past + 1000], 1, 16, 64, seed=past, spare_width=512)
    b.append([past])
    b.append([1000])
    b.check_attend([1000], 2, max_new=96)


def test_a_short_sequence_beside_a_prompt_takes_no_time():
    """A sequence with fewer key tiles than a prompt's are shared out to: its empty shares wait for nothing."""
    b = Batch(tsd, [2000, 9], 1, 16, 64, seed=2)
    b.append([2000, 9])
    q, both = b.rows(2009, 1), b.args([2000, 9])
    alone = {**both, "slots": both["slots"][:1].contiguous(), "starts": both["starts"][:2].contiguous()}
    ms = []
    for rows, a in ((2000, alone), (2009, both)):
        times = []
        for _ in range(8):
            x, y = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            x.record()
            b.cache.attend(q[:rows], **a, max_new=2000, max_len=2000)
            y.record()
            y.synchronize()
            times.append(x.elapsed_time(y))
        ms.append(min(times))
    assert ms[1] < ms[0] + 0.1, ms


def test_row_tiles_of_spoilt_rows_and_blocks():
    """NaN reaches the rows that see it in the tiled form too, and a bad sequence is all NaN."""
    b = Batch(tsd, [400, 300], 1, 16, 64, seed=3)
    k, v = b.rows(700, 1), b.rows(700, 1)
    v[100, 0, 2] = math.nan  # block 6 of sequence 0
    b.append([400, 300], k=k, v=v)
    a = b.args([400, 300])
    q = b.rows(700, 2)
    q[250, 1, 0] = math.inf
    out = b.cache.attend(q, window=120, sinks=3, max_new=400, **a)
    pos = torch.arange(400)
    bad = torch.zeros(700, 2, dtype=torch.bool)
    bad[:400][(pos >= 96) & (pos - 119 <= 111)] = True
    bad[250, 1] = True
    assert torch.equal(torch.isnan(out).all(2).cpu(), bad) and torch.equal(torch.isnan(out).any(2).cpu(), bad)
    t = b.table.clone()
    t[b.slots[1], 2] = b.cache.n_blocks
    out = b.cache.attend(q[400:], max_new=300, **{**a, "table": t, "slots": a["slots"][1:].contiguous(),
                                                  "starts": torch.tensor([0, 300], dtype=torch.int32, device="cuda")})
    assert bool(torch.isnan(out[32:]).all()) and not bool(torch.isnan(out[:32]).any())
    lens = a["lens"].clone()
    lens[b.slots[1]] = 299
    out2 = b.cache.attend(q, window=120, sinks=3, max_new=400, **{**a, "lens": lens})
    assert bool(torch.isnan(out2[400:]).all()) and torch.equal(torch.isnan(out2[:400]).all(2).cpu(), bad[:400])


@pytest.mark.parametrize("dim", [64, 128])
def test_long_contexts_over_several_ctas(dim):
    """Contexts split over CTAs and joined; the largest value at the far end, and scores of a wide range."""
    lens = [4000, 33, 2500]
    b = Batch(tsd, lens, 1, 32, dim, seed=dim)
    k, v = b.rows(sum(lens), 1), b.rows(sum(lens), 1)
    v[3] = 90.0
    k[3] *= 6
    b.append(lens, k=k, v=v)
    b.check_attend([1, 1, 1], 4)
    b.check_attend([1, 1, 1], 4, scale=1.0)
    b.check_attend([3, 0, 2], 2, window=3000, sinks=4)


@pytest.mark.parametrize("heads,count", [(1, 1), (12, 1), (1, 20), (5, 11)])
def test_long_contexts_of_other_row_counts(heads, count):
    """One and two column tiles of eight rows, row tiles of 32 and 64, each over several CTAs."""
    b = Batch(tsd, [3000 + count, 700], 1, 16, 64, seed=heads)
    b.append([3000, 700 - count])
    b.append([count, count])
    for kw in (dict(), dict(max_new=count, max_len=3000 + count)):
        b.check_attend([count, count], heads, **kw)


def test_many_short_contexts():
    """More sequences and key heads than the GPU runs CTAs at once."""
    lens = [1 + (37 * i) % 90 for i in range(260)]
    b = Batch(tsd, lens, 2, 16, 64, seed=4)
    b.append(lens)
    for heads in (2, 4, 20):
        b.check_attend([1] * len(lens), heads, max_len=90)


@pytest.mark.parametrize("counts,heads", [([1, 1], 2), ([9, 20], 4), ([50, 30], 1), ([300, 140], 2)])
def test_scores_that_grow(counts, heads):
    """Scores (below 44) that rise along the keys, by jumps inside a tile too, and fall again: the
    running maximum moves many times.  Negative scales turn rises into falls."""
    past = [400, 90]
    b = Batch(tsd, [p + c for p, c in zip(past, counts)], 1, 16, 64, seed=heads)
    n = sum(past) + sum(counts)
    t = torch.arange(n) % (n // 3)
    along = 0.25 * (t / 40 + 4 * (t % 97 > 50) + 0.3 * torch.randn(n, generator=b.g)).clamp(-12, 12)
    k = (along[:, None, None] * torch.ones(64)).to(b.dtype).cuda()
    b.append(past, k=k[:sum(past)])
    b.append(counts, k=k[sum(past):])
    q = (1 + 0.2 * b.rows(sum(counts), heads)).to(b.dtype)
    top = 0.125 * float(q.double().sum(2).abs().max()) * float(k.abs().max())
    assert top < 44
    for scale in (0.125, -0.125):
        b.check_attend(counts, heads, q=q, scale=scale)
    b.check_attend(counts, heads, q=q, scale=0.0)


def test_values_of_very_different_scales():
    """Blocks of values between 2^-20 and 2^20, the small ones with the larger weights too, and blocks of zeros."""
    for seed in range(3):
        b = Batch(tsd, [200], 1, 16, 64, seed=seed)
        k, v = b.rows(200, 1), b.rows(200, 1)
        for i in range(0, 200, 16):
            v[i:i + 16] *= 2.0 ** (((i // 16) * 7 + seed * 5) % 41 - 20)
        v[32:48] = 0
        b.append([200], k=k, v=v)
        b.check_attend([1], 2)
        b.check_attend([30], 2)


def test_extreme_queries():
    """Queries of zeros, tiny and large magnitude, one dominating element; a NaN or an infinity spoils its row alone."""
    b = Batch(tsd, [50], 1, 16, 64, seed=2)
    b.append([50])
    q = b.rows(8, 2)
    q[0] = 0
    q[1] *= 1e-30
    q[2] *= 8
    q[3, :, 1:] *= 1e-4
    q[4] = 1e-39
    b.check_attend([8], 2, q=q)
    q[5, 0, 7] = math.nan
    q[6, 1, 0] = -math.inf
    out = b.cache.attend(q, **b.args([8]))
    bad = torch.zeros(8, 2, dtype=torch.bool)
    bad[5, 0] = bad[6, 1] = True
    assert torch.equal(torch.isnan(out).any(2).cpu(), bad) and torch.equal(torch.isnan(out).all(2).cpu(), bad)


@pytest.mark.parametrize("heads", [2, 8])
def test_spoilt_blocks_reach_only_rows_that_see_them(heads):
    """A non-finite key or value makes the results NaN of rows that see a token of its block, in its head, and no others."""
    for which in ("k", "v"):
        b = Batch(tsd, [64], 2, 16, 64, seed=3)
        k, v = b.rows(64, 2), b.rows(64, 2)
        (k if which == "k" else v)[40, 1, 2] = math.inf  # block 2 (tokens 32..47) of head 1
        b.append([64], k=k, v=v)
        out = b.cache.attend(b.rows(64, heads), **b.args([64]), window=10, sinks=2)
        pos = torch.arange(64)
        sees = (pos >= 32) & (pos - 9 <= 47)
        bad = torch.zeros(64, heads, dtype=torch.bool)
        bad[sees, heads // 2:] = True
        assert torch.equal(torch.isnan(out).all(2).cpu(), bad) and torch.equal(torch.isnan(out).any(2).cpu(), bad), which


def test_bad_blocks_slots_and_lengths():
    """Block ids out of the pool, slots and lengths out of range: NaN for the rows concerned, nothing else touched."""
    b = Batch(tsd, [40, 40, 40], 1, 16, 64, seed=4)
    b.append([40, 40, 40])
    a = b.args([2, 2, 2])
    q = b.rows(6, 2)
    good = b.cache.attend(q, **a)

    def spoilt(rows, **change):
        for c in (dict(), dict(max_new=1, max_len=5), dict(max_new=2)):
            out = b.cache.attend(q, **{**a, **change}, **c)
            bad = torch.zeros(6, dtype=torch.bool)
            bad[rows] = True
            assert torch.equal(torch.isnan(out).flatten(1).all(1).cpu(), bad), (rows, change.keys())
            assert torch.equal(out[~bad], good[~bad]) or float((out[~bad] - good[~bad]).abs().max()) < 0.02

    for bad_id in (-1, b.cache.n_blocks, 2 ** 31 - 1, -2 ** 31):
        t = b.table.clone()
        t[b.slots[1], 1] = bad_id
        spoilt([2, 3], table=t)
        k, v = b.cache.read(rows=6, **{**a, "table": t})
        assert not bool(torch.isnan(k).any())  # the last tokens are in block 2
        t[b.slots[1], 2] = bad_id
        k, v = b.cache.read(rows=6, **{**a, "table": t})
        assert bool(torch.isnan(k[2:4]).all()) and not bool(torch.isnan(k[[0, 1, 4, 5]]).any())
        before = b.cache.k.clone()
        b.cache.append(b.rows(6, 1), b.rows(6, 1), **{**a, "table": torch.full_like(t, bad_id)})
        assert torch.equal(before, b.cache.k)
        b.cache.k_tail.zero_(), b.cache.v_tail.zero_()
    for bad_len in (-1, 1, 2 ** 30, b.table.shape[1] * 16 + 1):
        lens = a["lens"].clone()
        lens[b.slots[2]] = bad_len
        spoilt([4, 5], lens=lens)
        before = b.cache.k.clone()
        only = torch.tensor([b.slots[2]], dtype=torch.int32, device="cuda")
        b.cache.append(b.rows(2, 1), b.rows(2, 1), table=b.table, lens=lens, slots=only,
                       starts=torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
        assert torch.equal(before, b.cache.k)
    for bad_slot in (-1, b.cache.n_slots, 2 ** 31 - 1):
        slots = a["slots"].clone()
        slots[0] = bad_slot
        spoilt([0, 1], slots=slots)
    starts = a["starts"].clone()
    starts[3] = 100  # more rows than the call has, and than the sequence has tokens
    spoilt([4, 5], starts=starts)
    starts = torch.tensor([-5, 2, 4, 6], dtype=torch.int32, device="cuda")
    spoilt([0, 1], starts=starts)


def test_rows_behind_the_last_sequence_stay():
    b = Batch(tsd, [600, 40], 1, 16, 64, seed=4)
    b.append([600, 40])
    for counts in ([1, 1], [3, 9]):
        n = sum(counts)
        q = b.rows(n + 6, 4)
        out = torch.full((n + 6, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        b.cache.attend(q, out=out, **b.args(counts))
        assert bool((out[n:] == 7).all())
        b.compare(out, q, counts, 0, 0, 64 ** -0.5)


def test_defaults_one_row_each_in_slot_order():
    lens = [5, 77, 30]
    b = Batch(tsd, lens, 2, 16, 64, seed=1, spare_slots=0)
    b.append(lens)
    q = b.rows(3, 2)
    a = b.args([1, 1, 1])
    order = torch.argsort(a["slots"])  # sequence i of the call below is slot i
    out = b.cache.attend(q, a["table"], a["lens"])
    ref = b.cache.attend(q[a["slots"].long()], **a)
    assert torch.equal(out, ref[order])


def test_sizes_past_32_bits():
    """Windows and sinks that no sequence reaches are as none, and sizes that 32 bits would cut are refused."""
    b = Batch(tsd, [90, 200], 1, 16, 64, seed=1)
    b.append([90, 200])
    a = b.args([3, 100])
    q = b.rows(103, 2)
    want = b.cache.attend(q, **a, max_new=100)
    for window, sinks in ((2 ** 40, 0), (2 ** 32 + 5, 2 ** 32 + 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert torch.equal(b.cache.attend(q, **a, window=window, sinks=sinks, max_new=100), want)
    assert torch.equal(b.cache.attend(q, **a, window=7, sinks=2 ** 33, max_new=2 ** 40), want)
    with pytest.raises(ValueError, match="rows"):
        b.cache.read(rows=2 ** 32 + 1, **a)


def test_same_slot_twice_in_attention():
    b = Batch(tsd, [40, 50], 1, 16, 64, seed=1)
    b.append([40, 50])
    a = b.args([1, 1])
    a["slots"] = a["slots"][[0, 0]].contiguous()
    q = b.rows(1, 2).repeat(2, 1, 1)
    out = b.cache.attend(q, **a)
    assert torch.equal(out[0], out[1])


def test_results_do_not_depend_on_the_hints():
    """max_new and max_len wrong in either direction: the same up to the sums' order."""
    b = Batch(tsd, [900, 3, 200], 1, 16, 64, seed=9)
    b.append([880, 0, 199])
    b.append([20, 3, 1], max_new=1)
    b.check_held()
    q = b.rows(24, 2)
    for kw in (dict(), dict(max_new=1), dict(max_new=24, max_len=16), dict(max_new=1000000, max_len=2 ** 31 - 1)):
        b.check_attend([20, 3, 1], 2, q=q, **kw)


# ---------------------------------------------------------------- as programs call them

def test_a_captured_decode_loop():
    """One graph of append and attention, replayed while lengths grow on the device; the same bits as direct calls."""
    b, c = (Batch(tsd, [120, 60, 33], 2, 16, 64, seed=5) for _ in range(2))
    for x in (b, c):
        x.g.manual_seed(1)
        x.append([100, 40, 13])
    ks, vs, qs = (torch.stack([b.rows(3, h) for _ in range(20)]) for h in (2, 2, 8))
    a = c.args([1, 1, 1])
    k, v, q = ks[0].clone(), vs[0].clone(), qs[0].clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        c.cache.append(k, v, **a, max_new=1)
        out = c.cache.attend(q, **a, max_new=1)
    for i in range(20):
        k.copy_(ks[i]), v.copy_(vs[i]), q.copy_(qs[i])
        a["lens"][a["slots"].long()] += 1
        graph.replay()
        b.append([1, 1, 1], k=ks[i], v=vs[i], max_new=1)
        ref = b.cache.attend(qs[i], **b.args([1, 1, 1]), max_new=1)
        assert torch.equal(out, ref), i
    b.check_attend([1, 1, 1], 8)


def test_two_streams_at_once():
    b = Batch(tsd, [3000, 700], 1, 32, 128, seed=5)
    b.append([3000, 700])
    a = b.args([1, 1])
    qs = [b.rows(2, 8) for _ in range(2)]
    want = [b.cache.attend(q, **a) for q in qs]
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = [b.cache.attend(qs[i], **a, stream=s[i]) for i in range(2)]
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_offsets_past_32_bits():
    """A pool whose byte offsets pass 2^32: its last blocks, and queries at the end of a wide table."""
    block, dim, heads = 64, 128, 8
    per = heads * block * dim
    n_blocks = (1 << 32) // per + 64
    cache = tsd.KV8Cache.empty(n_blocks, 1, heads, dim, block=block)
    width = 8
    ids = torch.arange(n_blocks - width, n_blocks, dtype=torch.int32)[None]
    b = Batch(tsd, [500], heads, block, dim, seed=1, spare_slots=0, spare_width=0)
    b.cache, b.table = cache, ids.cuda()
    b.append([500])
    b.check_held(tail=40)
    b.check_attend([1], heads)
    b.check_attend([70], heads)


def test_a_language_models_step():
    """A small attention language model over streams: prompts, then single tokens
    chosen by the scores; every step's cache, attention and scores against fp64."""
    H, heads, kv, dim, C = 128, 4, 2, 64, 300
    g = torch.Generator().manual_seed(0)
    emb = (torch.randn(C, H, generator=g)).to(torch.bfloat16).cuda()
    wqkv = (torch.randn(H, (heads + 2 * kv) * dim, generator=g) * H ** -0.5).to(torch.bfloat16).cuda()
    wo = (torch.randn(heads * dim, H, generator=g) * 0.1).to(torch.bfloat16).cuda()
    wt = ((torch.randn(C, H, generator=g) * 0.1) * 256).round().div(256).to(torch.bfloat16).cuda()
    counts = [70, 1, 20]
    b = Batch(tsd, [110, 41, 60], kv, 16, dim, seed=2)
    tokens = torch.randint(0, C, (sum(counts),), generator=g).cuda()
    for step in range(12):
        x = emb[tokens]
        qkv = (x @ wqkv).view(-1, heads + 2 * kv, dim)
        b.append(counts, k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:])
        b.check_held()
        att = b.check_attend(counts, heads, q=qkv[:, :heads], window=40, sinks=4)
        last = torch.cumsum(torch.tensor(counts), 0) - 1
        h = (x[last] + att.reshape(len(x), -1)[last] @ wo)
        r = tsd.joint_label_scores(h, wt, k=3)
        lp = torch.log_softmax(h.double() @ wt.double().t(), 1)
        top = lp.max(1)
        assert float((r.alt_logp[:, 0] - top.values).abs().max()) < 1e-4
        again = tsd.joint_label_scores(h, wt, r.alt_labels.contiguous(), k=3)
        assert torch.equal(again.logp, r.alt_logp)
        tokens = r.alt_labels[:, 0].long()
        counts = [1, 1, 1]
