"""label_scores (logits in memory) and joint_label_scores (joint rows times
output weights) against a plain 64-bit computation: sizes around every change
of variant, types, strides and alignments, masks, ties, non-finite logits, and
the calls that a program makes of them (other streams, captured graphs)."""
import math

import pytest
import torch

import paper_2609_14991_gb300 as tsd
from tests import label_util as lu

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def rows(n, C, dtype, seed, ld=None, offset=0, scale=3.0):
    """[n, C] logits: a view of a wider buffer, `offset` elements in."""
    g = torch.Generator().manual_seed(seed)
    ld = ld or C
    buf = (torch.randn(n * ld + offset + 8, generator=g) * scale).to(TYPES[dtype]).to(DEV)
    return buf[offset:offset + n * ld].view(n, ld)[:, :C]


def given(n, m, C, seed):
    g = torch.Generator().manual_seed(seed + 1)
    lab = torch.randint(0, C, (n, m), generator=g, dtype=torch.int32)
    if m and n > 1:
        lab[n // 2, 0] = -1
    return lab


def check(x, lab, k, temperature=1.0, what=""):
    got = tsd.label_scores(x, None if lab is None else lab.to(DEV), k=k, temperature=temperature)
    want = lu.oracle(x.double().cpu(), lab, k, temperature)
    fin = x.double()[torch.isfinite(x.double())]
    spread = float(fin.max() - fin.min()) / temperature if fin.numel() else 0.0
    lu.assert_scores(got, want, what, spread)
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [1, 2, 5, 7, 31, 127, 129, 255, 256, 257, 263, 1023, 1024, 1025, 1031, 2049, 4097, 8193, 8200])
def test_sizes(C, dtype):
    n = 5 if C < 3000 else 2
    check(rows(n, C, dtype, C), given(n, 2, C, C), min(5, 8), what=(C, dtype))


@pytest.mark.parametrize("dtype,C", [("fp32", 16385), ("fp32", 32769), ("bf16", 40001), ("fp16", 65537), ("bf16", 131073),
                                     ("fp32", 131079), ("fp32", 262144), ("bf16", 262143)])
def test_wide_rows(dtype, C):
    """Rows of a cluster of 2, 4 and 8 CTAs, and of 64 logits per thread."""
    check(rows(2, C, dtype, 3, ld=C + 3, offset=1), given(2, 1, C, 5), 8, temperature=0.7, what=(C, dtype))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (7, 1)])
def test_strides_and_alignment(offset, pad, dtype):
    for C in (3, 66, 1030):
        check(rows(9, C, dtype, 7 * offset + pad, ld=C + pad, offset=offset), given(9, 3, C, 11), 4, what=(C, dtype, offset, pad))


@pytest.mark.parametrize("m,k", [(0, 0), (0, 8), (8, 0), (1, 1), (8, 8)])
def test_counts_of_labels_and_alternatives(m, k):
    check(rows(7, 300, "fp32", 2), given(7, m, 300, 2) if m else None, k, what=(m, k))


def test_temperature():
    for t in (0.1, 0.7, 2.5, 100.0):
        check(rows(6, 500, "fp32", 3), given(6, 2, 500, 3), 3, temperature=t, what=t)


@pytest.mark.parametrize("C", [9, 300, 5000, 70001])
def test_masks(C):
    """Some, most, all but one, and all labels masked; fewer labels than alternatives."""
    x = rows(6, C, "fp32", 9)
    x[1, ::3] = -math.inf
    x[2, 1:] = -math.inf
    x[3] = -math.inf
    x[4, :-4] = -math.inf
    x[5, : C // 2] = -math.inf
    lab = given(6, 2, C, 9)
    lab[2, 0], lab[2, 1] = 0, 1
    check(x, lab, 8, what=C)


@pytest.mark.parametrize("C", [8, 333, 4096, 40000])
def test_ties(C):
    """Equal logits everywhere (more than are gathered), in half of the row, and -0 beside 0."""
    x = rows(5, C, "fp32", 4)
    x[0] = 1.5
    x[1] = (x[1] * 0.5).round()
    x[2] = 0.0
    x[2, 1::2] = -0.0
    x[3] = torch.arange(C, device=DEV).float()
    x[4] = -torch.arange(C, device=DEV).float()
    check(x, given(5, 1, C, 4), 8, what=C)


def test_sorted_rows_gather_nothing_twice():
    """Descending runs put the largest logits into few threads."""
    for C in (1024, 4096, 16384):
        x = torch.linspace(30, -30, C).repeat(3, 1).to(DEV)
        x[1] = x[1].flip(0)
        x[2] = x[2].view(-1, 32).t().reshape(-1)
        check(x.contiguous(), given(3, 1, C, 1), 8, what=C)


@pytest.mark.parametrize("C", [5, 700, 9000, 50000])
def test_non_finite(C):
    x = rows(5, C, "fp32", 6)
    x[0, C // 2] = math.nan
    x[1, 0] = math.inf
    x[2] = math.nan
    x[3, C - 1] = -math.inf
    lab = given(5, 2, C, 6)
    check(x, lab, 3, what=C)


def test_large_offsets_cost_no_precision():
    x = rows(4, 1000, "fp32", 8)
    base = tsd.label_scores((x * 8).round() / 8, k=3)
    far = tsd.label_scores((x * 8).round() / 8 + 65536.0, k=3)  # exact in fp32
    assert torch.equal(base.alt_labels, far.alt_labels)
    assert torch.equal(base.alt_logp, far.alt_logp) and torch.equal(base.entropy, far.entropy)


def test_labels_outside_the_row():
    x = rows(3, 50, "fp32", 1)
    lab = torch.tensor([[-1, 50], [-2, 49], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32)
    got = check(x, lab, 0)
    assert torch.isnan(got.logp[2]).all() and got.logp[0, 0] == 0


def test_rows_do_not_depend_on_the_call():
    x = rows(300, 1025, "fp32", 12)
    lab = given(300, 2, 1025, 12).to(DEV)
    all_ = tsd.label_scores(x, lab, k=4)
    for r in (0, 7, 299):
        one = tsd.label_scores(x[r:r + 1], lab[r:r + 1], k=4)
        assert torch.equal(one.logp[0], all_.logp[r]) and torch.equal(one.entropy[0], all_.entropy[r])
        assert torch.equal(one.alt_labels[0], all_.alt_labels[r]) and torch.equal(one.alt_logp[0], all_.alt_logp[r])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C,n", [(37, 2000), (263, 700), (1031, 1300), (4099, 400), (20001, 40), (70001, 9)])
def test_bits_do_not_depend_on_other_rows(C, n, dtype):
    """Rows of any alignment, alone and a few of them at a time, at the addresses that they have in a large call."""
    x = rows(n, C, dtype, C, offset=3)
    lab = given(n, 2, C, C).to(DEV)
    all_ = tsd.label_scores(x, lab, k=5, temperature=0.9)
    for a, b in [(0, 1), (1, 2), (n - 1, n), (3, 8), (n // 2, n)]:
        some = tsd.label_scores(x[a:b], lab[a:b], k=5, temperature=0.9)
        for name in ("logp", "entropy", "alt_labels", "alt_logp"):
            one, other = getattr(some, name), getattr(all_, name)[a:b]
            assert torch.equal(torch.nan_to_num(one, nan=7.0), torch.nan_to_num(other, nan=7.0)), (name, a, b)  # (NaN: a label outside the row)


# ---------------------------------------------------------------- from joint rows

def joint_inputs(n, H, C, seed, lda=None, ldw=None):
    """Activations and weights on a grid on which every product and sum is exact in
    fp32: multiples of 1/16 below 8 times multiples of 1/256 below 1/4 are
    multiples of 2^-12 below 2, H <= 2048 of them below 2^12, 24 bits."""
    g = torch.Generator().manual_seed(seed)
    a = (torch.relu(torch.randn(n, lda or H, generator=g) * 1.4).clamp(max=7.9) * 16).round() / 16
    w = (torch.randn(C, ldw or H, generator=g) * 0.07).clamp(-0.24, 0.24)
    w = (w * 256).round() / 256
    return a.to(torch.bfloat16).to(DEV)[:, :H], w.to(torch.bfloat16).to(DEV)[:, :H]


def check_joint(n, H, C, m, k, temperature=1.0, seed=0, **ld):
    A, W = joint_inputs(n, H, C, seed, **ld)
    lab = given(n, m, C, seed) if m else None
    got = tsd.joint_label_scores(A, W, None if lab is None else lab.to(DEV), k=k, temperature=temperature)
    x = A.double().cpu() @ W.double().cpu().t()
    lu.assert_scores(got, lu.oracle(x, lab, k, temperature), (n, H, C, m, k), float(x.max() - x.min()) / temperature)


@pytest.mark.parametrize("n,H,C", [(1, 64, 1), (1, 64, 17), (3, 128, 64), (2, 320, 65), (7, 320, 257), (64, 64, 128),
                                   (127, 192, 129), (128, 256, 31), (129, 64, 1025), (40, 1024, 300), (5, 2048, 70)])
def test_joint_sizes(n, H, C):
    check_joint(n, H, C, 2, 4, seed=n + C)


@pytest.mark.parametrize("n,C", [(300, 2000), (1300, 1025), (2500, 2049), (5000, 1000), (2000, 4097), (2600, 4097),
                                 (9001, 1025), (20000, 513), (40000, 60), (129, 40001)])
def test_joint_tile_shapes(n, C):
    """Calls that store their logits (128 x 64, 128 x 128 and paired tiles) and calls that do not, one row tile over
    several workers (up to all of them) and several row tiles over one: every row against the 64-bit sums, the
    labels exactly."""
    A, W = joint_inputs(n, 128, C, n)
    lab = given(n, 2, C, n)
    for k in (0, 3, 8):
        got = tsd.joint_label_scores(A, W, lab.to(DEV), k=k, temperature=1.3)
        x = A.double() @ W.double().t()
        lp = torch.log_softmax(x / 1.3, 1)
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        logp = torch.where(lab.to(DEV) < 0, 0.0, torch.gather(lp, 1, lab.to(DEV).clamp(min=0).long()))
        want = (logp.cpu(), -(lp.exp() * lp).sum(1).cpu(), order.to(torch.int32).cpu(), torch.gather(lp, 1, order).cpu())
        lu.assert_scores(got, want, (n, C, k), float(x.max() - x.min()) / 1.3)


@pytest.mark.parametrize("m,k", [(0, 0), (0, 1), (8, 0), (8, 8), (1, 5)])
def test_joint_counts(m, k):
    check_joint(70, 128, 90, m, k, seed=3)


def test_joint_strides():
    check_joint(33, 128, 140, 2, 4, lda=136, ldw=256)
    check_joint(300, 64, 5000, 2, 4, lda=72, ldw=64)


def test_joint_ties_and_equal_rows():
    """All weights equal: every logit equal, the lowest labels in order; a label outside the row.  Then few
    distinct weights, so that every logit occurs many times, in runs and scattered, and ascending ones, so
    that every logit is the best so far."""
    for n, C in ((130, 1000), (130, 40000), (5000, 2100)):
        H = 64
        A, W1 = joint_inputs(n, H, C, 1)
        W = W1[:1].repeat(C, 1).contiguous()
        lab = torch.tensor([[C]] * n, dtype=torch.int32, device=DEV)
        for k in (3, 8):
            got = tsd.joint_label_scores(A, W, lab, k=k)
            assert torch.equal(got.alt_labels.cpu(), torch.arange(k, dtype=torch.int32).repeat(n, 1))
            # all logits are the largest, so every sum counts exact ones
            assert float((got.alt_logp + math.log(C)).abs().max()) < 1e-5
            assert float((got.entropy - math.log(C)).abs().max()) < 2e-5
            assert torch.isnan(got.logp).all()
        g = torch.Generator().manual_seed(3)
        for order in (torch.arange(C) // 37 % 23, torch.randint(0, 23, (C,), generator=g), torch.arange(C) * 23 // C):
            order = order.to(DEV)
            W = (W1[:23].sort(0).values[order] if order[0] == 0 and order[-1] == 22 else W1[:23][order]).contiguous()
            got = tsd.joint_label_scores(A, W, None, k=8)
            x = A.double() @ W.double().t()
            want = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :8].to(torch.int32)
            assert torch.equal(got.alt_labels, want), (n, C)


def test_joint_ascending_logits():
    """Every later label is better: the buffers of candidates run full again and again."""
    n, H, C = 700, 64, 20000
    A = torch.zeros(n, H, dtype=torch.bfloat16, device=DEV)
    A[:, 0], A[:, 1] = 1, 1
    i = torch.arange(C)
    W = torch.zeros(C, H)
    W[:, 0], W[:, 1] = i // 128, (i % 128) / 128  # bf16 holds both parts, fp32 their sum
    got = tsd.joint_label_scores(A, W.to(torch.bfloat16).to(DEV), None, k=8)
    assert torch.equal(got.alt_labels.cpu(), torch.arange(C - 1, C - 9, -1, dtype=torch.int32).repeat(n, 1))
    got = tsd.joint_label_scores(A, W.flip(0).to(torch.bfloat16).to(DEV), None, k=8)
    assert torch.equal(got.alt_labels.cpu(), torch.arange(8, dtype=torch.int32).repeat(n, 1))


@pytest.mark.parametrize("n,C", [(260, 300), (260, 30000)])
def test_joint_non_finite_rows(n, C):
    A, W = joint_inputs(n, 64, C, 2)
    A[3, 5] = math.nan
    A[200, 0] = math.inf
    got = tsd.joint_label_scores(A, W, torch.zeros(n, dtype=torch.int32, device=DEV), k=2)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[3] = bad[200] = True
    assert torch.equal(torch.isnan(got.logp).cpu(), bad) and torch.equal(torch.isnan(got.entropy).cpu(), bad)
    assert torch.equal((got.alt_labels == -1).all(1).cpu(), bad) and torch.equal(torch.isnan(got.alt_logp).all(1).cpu(), bad)


def test_joint_agrees_with_the_decoders_selection():
    """The best alternative and its score are joint_select_noalloc's without a bias."""
    n, H, V = 100, 320, 256
    A, W = joint_inputs(n, H, V + 1, 5)
    lab = torch.empty(n, dtype=torch.int32, device=DEV)
    sc = torch.empty(n, dtype=torch.float32, device=DEV)
    tsd.joint_select_noalloc(A, W.view(torch.int16), None, lab, sc)
    got = tsd.joint_label_scores(A, W, lab, k=1)
    assert torch.equal(got.alt_labels[:, 0], lab)
    assert float((got.alt_logp[:, 0] - sc).abs().max()) < 2e-5
    assert torch.equal(got.logp, got.alt_logp[:, 0])


# ---------------------------------------------------------------- as programs call them

def test_streams_and_graphs():
    """On another stream, two calls at once on two streams, and captured: replays read new inputs."""
    A, W = joint_inputs(200, 128, 500, 4)
    A2, _ = joint_inputs(200, 128, 500, 5)
    x = rows(50, 900, "fp32", 4)
    lab = given(200, 1, 500, 4).to(DEV)
    want, want2 = (tsd.joint_label_scores(a, W, lab, k=3) for a in (A, A2))
    want_x = tsd.label_scores(x, k=3)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        g1 = tsd.joint_label_scores(A, W, lab, k=3, stream=s1)
        g2 = tsd.joint_label_scores(A2, W, lab, k=3, stream=s2)
        g3 = tsd.label_scores(x, k=3, stream=s2)
    torch.cuda.synchronize()
    for g, w in ((g1, want), (g2, want2), (g3, want_x)):
        for f in ("logp", "entropy", "alt_labels", "alt_logp"):
            assert torch.equal(getattr(g, f), getattr(w, f)), f
    buf = A.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = tsd.joint_label_scores(buf, W, lab, k=3)
        out_x = tsd.label_scores(x, k=3)
    for a, w in ((A, want), (A2, want2), (A, want)):
        buf.copy_(a)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.logp, w.logp) and torch.equal(out.alt_labels, w.alt_labels)
        assert torch.equal(out_x.entropy, want_x.entropy)


def test_given_outputs_and_rows_behind():
    x = rows(10, 100, "fp32", 2)
    lab = given(10, 1, 100, 2).to(DEV)
    out = tsd.LabelScores(torch.full((4, 1), 7.0, device=DEV), torch.full((4,), 7.0, device=DEV),
                          torch.full((4, 2), 7, dtype=torch.int32, device=DEV), torch.full((4, 2), 7.0, device=DEV))
    got = tsd.label_scores(x[:4], lab[:4], k=2, out=out)
    assert got is out and torch.equal(out.logp, tsd.label_scores(x, lab, k=2).logp[:4])


def test_refusals_on_the_device():
    x = rows(4, 10, "fp32", 0)
    for bad in (dict(k=9), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=-1.0)):
        with pytest.raises((ValueError, tsd.TsdError)):
            tsd.label_scores(x, **bad)
    with pytest.raises(ValueError, match="adjacent"):
        tsd.label_scores(x.t())
    with pytest.raises(ValueError, match="labels"):
        tsd.label_scores(x, torch.zeros(3, dtype=torch.int32, device=DEV))
    A, W = joint_inputs(4, 64, 10, 0)
    with pytest.raises(tsd.TsdError, match="multiple of 64"):
        tsd.joint_label_scores(A[:, :32], W[:, :32])
    with pytest.raises(tsd.TsdError, match="strides"):
        tsd.joint_label_scores(torch.zeros(4, 65, dtype=torch.bfloat16, device=DEV)[:, :64], W)
