"""label_scores on long rows: equal best logits, few and many, spread and close together."""
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
