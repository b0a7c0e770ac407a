"""label_scores on long rows: equal best logits, few and many, spread and close together; rows
around the most that each variant holds."""
import math

import pytest
import torch

import paper_2609_14991_gb300 as tsd
from tests import label_util as lu

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EQUAL = (9, 32, 33, 64, 65, 90, 100, 128, 129, 300)


def places(count, C, how):
    """Ascending labels of `count` equal logits."""
    i = torch.arange(count)
    if how == "spread":
        return i * (C // count) + 3
    if how == "near":  # in the vectors of the first CTA of a cluster, no two in one
        return i * 15 + 1
    if how == "dense":
        return i + C // 3
    return C - count + i  # "end"


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [5000, 9001, 20000, 40000, 65537, 131073, 262144])
def test_equal_best_logits(C, dtype):
    """Every count and place, as rows of one call: the lowest labels in order, and the sums."""
    g = torch.Generator().manual_seed(C)
    kinds = [(n, how) for n in EQUAL for how in ("spread", "near", "dense", "end")]
    x = (torch.randn(len(kinds), C, generator=g).clamp(-2, 2)).to(TYPES[dtype])
    for r, (n, how) in enumerate(kinds):
        x[r, places(n, C, how)] = 4.0
    lab = torch.randint(0, C, (len(kinds), 1), generator=g, dtype=torch.int32)
    for k in (1, 8):
        got = tsd.label_scores(x.to(DEV), lab.to(DEV), k=k)
        lu.assert_scores(got, lu.oracle(x.double(), lab, k), (C, dtype, k), 6.0)


@pytest.mark.parametrize("C", [20000, 40000, 262144])
def test_a_few_better_ones_above_equal_ones(C):
    """The best logits in order, then the first of many equal ones; all else masked."""
    x = torch.full((len(EQUAL), C), -math.inf)
    for r, n in enumerate(EQUAL):
        x[r, places(n, C, "spread")] = 1.0
        x[r, [C - 1, 0, C // 2]] = torch.tensor([3.0, 2.0, 2.0])
    got = tsd.label_scores(x.to(DEV), k=8)
    lu.assert_scores(got, lu.oracle(x.double(), None, 8), C, 2.0)


def test_joint_equal_best_logits():
    """The same from joint rows whose logits are stored."""
    H, C = 64, 20000
    g = torch.Generator().manual_seed(1)
    A = torch.ones(2, H, dtype=torch.bfloat16)
    for n in EQUAL:
        W = (torch.randn(C, H, generator=g).clamp(-2, 2) / 64).mul(64).round().div(64)
        W[places(n, C, "spread")] = 0.5
        x = A.double() @ W.double().t()
        got = tsd.joint_label_scores(A.to(DEV), W.to(torch.bfloat16).to(DEV), k=8)
        lu.assert_scores(got, lu.oracle(x, None, 8), n, float(x.max() - x.min()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("threads", [32, 64, 128, 256, 512, 1024, 2048, 4096])
def test_rows_around_what_a_variant_holds(threads, dtype):
    """Aligned rows of as many whole vectors as that many threads hold (in 8, 32 and 64 logits each), up
    to eight more, and the vectors' ends: the largest logit in the last whole vector, the next in the end."""
    size = torch.finfo(TYPES[dtype]).bits // 8
    vec = 16 // size
    for each in (8, 32, 64):
        full = threads * each
        for C in sorted({full + d for d in (-vec, -1, 0, 1)} | {full + d * vec + e for d in range(1, 9) for e in (0, vec - 1)}):
            if C > 262144:
                continue
            x = (torch.randn(2, -(-C // vec) * vec, device=DEV)).to(TYPES[dtype])[:, :C]
            assert x.data_ptr() % 16 == 0 and x.stride(0) % vec == 0
            last = C // vec * vec - 1
            x[0, last], x[0, last - vec + 1], x[1, C - 1], x[1, 0] = 20.0, 18.0, 20.0, 19.0
            got = tsd.label_scores(x, torch.tensor([[last], [C - 1]], dtype=torch.int32, device=DEV), k=2)
            lp = torch.log_softmax(x.double(), 1)
            top = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :2]
            assert torch.equal(got.alt_labels, top.to(torch.int32)), C
            # a logarithm of a sum near 1 and a difference of logits below 32: see assert_scores
            assert float((got.alt_logp - torch.gather(lp, 1, top)).abs().max()) < 8e-6 + 3 * 2 ** -24 * 32, C
            assert torch.equal(got.logp[:, 0], got.alt_logp[:, 0]), C


@pytest.mark.parametrize("n,C", [(3, 700), (5000, 2100), (129, 40001), (260, 30000)])
@pytest.mark.parametrize("temperature", [1.0, 0.1])
def test_joint_masks_of_the_types_lowest_value(n, C, temperature):
    """Labels ruled out by a column of bf16's lowest value, in half of the rows: runs of them and single ones
    (stored and kept logits).  Their weight is 0, and the others' scores are those of a row without them."""
    H, low = 64, torch.finfo(torch.bfloat16).min
    g = torch.Generator().manual_seed(C)
    A = ((torch.relu(torch.randn(n, H, generator=g) * 1.4).clamp(max=7.9) * 16).round() / 16)
    W = ((torch.randn(C, H, generator=g) * 0.07).clamp(-0.24, 0.24) * 256).round() / 256
    off = torch.rand(C, generator=g) < 0.1
    off[:300] = True  # whole tiles' parts from the first label on
    off[C // 2:C // 2 + 64] = True
    off[C - 5:] = True
    A[:, 0] = (torch.arange(n) % 3 != 1).float()
    W[:, 0] = off * low
    A, W = A.to(torch.bfloat16).to(DEV), W.to(torch.bfloat16).to(DEV)
    lab = torch.stack([torch.randint(0, C, (n,), generator=g), torch.full((n,), 7)], 1).to(torch.int32).to(DEV)
    x = A.double() @ W.double().t()
    lp = torch.log_softmax(x / temperature, 1)
    fine = x > -1e30
    spread = float((x[fine].max() - x[fine].min())) / temperature
    tol = 8e-6 + 3 * 2 ** -24 * spread  # as in assert_scores
    for k in (0, 4, 8):
        got = tsd.joint_label_scores(A, W, lab, k=k, temperature=temperature)
        assert float((got.entropy + (lp.exp() * lp).sum(1)).abs().max()) < 3 * tol, k
        want = torch.gather(lp, 1, lab.long())
        seen = torch.gather(fine, 1, lab.long())
        assert float((got.logp - want)[seen].abs().max()) < tol
        assert bool((got.logp[~seen] < -1e38).all())
        top = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(got.alt_labels, top.to(torch.int32))
        assert k == 0 or float((got.alt_logp - torch.gather(lp, 1, top)).abs().max()) < tol


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [40, 1025, 9000, 50000])
def test_masks_of_the_types_lowest_value(C, dtype):
    low = torch.finfo(TYPES[dtype]).min
    x = torch.randn(4, C, device=DEV).to(TYPES[dtype])
    x[1, : C // 2], x[2, 1:], x[3, ::3] = low, low, low
    lp = torch.log_softmax(x.double(), 1)
    got = tsd.label_scores(x, k=3)
    assert float((got.entropy + (lp.exp() * lp).sum(1)).abs().max()) < 3 * (8e-6 + 3 * 2 ** -24 * 16)
    top = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :3]
    assert torch.equal(got.alt_labels, top.to(torch.int32))
