"""Prompts in a sliding window over the 8-bit cache: rows of a tile whose window
begins steps after the first row's, keys split over CTAs and not, at weights far
from 1, against the plain 64-bit formulas."""
import math

import pytest
import torch

import paper_2609_14991_gb300 as tsd
from tests.kv8_util import Batch

pytestmark = pytest.mark.gpu


def check(b, counts, heads, window, sinks, q, scale=None, **kw):
    """Attention of counts[i] last tokens of each sequence, every row against 64 bits.

    Bounds, per result: a weight is rounded to fp16 (2^-11 of it) for the products and
    not for the sum that divides them.  In both it carries e: its exponent's error, at
    most eight roundings of 2^-23 of A (the sums of |q k| in units of log2, the cut of
    each k-step's sum among them, and 32 for the value scale's logarithm), times ln 2;
    and the sums' own, chains of below 256 fp32 additions, 2^-15.  So (2^-11 + 2 e)
    sum p |v|; weights below 2^-21 of the largest are fp16 subnormals, off by at most 2^-32 of
    it each; then half a step of the result's type."""
    scale = b.dim ** -0.5 if scale is None else scale
    out = b.cache.attend(q, **b.args(counts), window=window, sinks=sinks, scale=scale, **kw).double()
    g, at = heads // b.heads, 0
    for i, c in enumerate(counts):
        if not c:
            continue
        L = b.len[i]
        k, v = (b.model.held(x, b.slots[i]).cuda() for x in "kv")
        key, pos = torch.arange(L, device="cuda"), torch.arange(L - c, L, device="cuda")[:, None]
        see = key <= pos
        if window:
            see &= (key > pos - window) | (key < sinks)
        for h in range(heads):
            x, kk, vv = q[at:at + c, h].double(), k[:, h // g], v[:, h // g]
            p = torch.softmax(torch.where(see, x @ kk.t() * scale, -math.inf), 1)
            want, mag = p @ vv, p @ vv.abs()
            A = float((x.abs() @ kk.abs().t()).max()) * abs(scale) / math.log(2) + 32
            e = math.log(2) * 8 * 2 ** -23 * A + 2 ** -15
            tol = (2 ** -11 + 2 * e) * mag + L * 2 ** -32 * vv.abs().max() + torch.finfo(b.dtype).eps / 2 * want.abs()
            if b.dtype == torch.float16:
                tol += 2 ** -25  # its subnormals' half step
            off = (out[at:at + c, h] - want).abs()
            bad = ~(off <= tol).all(1)
            assert not bool(bad.any()), (i, h, int(bad.sum()), c, float((off / tol).max()))
        at += c


def fill(heads, counts, past, dim=64, dtype=torch.bfloat16, seed=0, spread=1.0, values=1.0, shift=0.0, block=16, kv=1):
    """A batch with its tokens, and queries of the new ones: queries and keys of that spread, scores
    shifted by about `shift` (a constant dimension), values times `values`."""
    b = Batch(tsd, [p + c for p, c in zip(past, counts)], kv, block, dim, dtype, seed=seed)
    side = math.sqrt(abs(shift) * math.sqrt(dim))

    def rows(n, h, s, sign):
        x = b.rows(n, h).float() * s
        if shift:
            x[..., 0] = sign * side
        return x.to(dtype)

    for cs in (past, counts):
        if sum(cs):
            n = sum(cs)
            b.append(cs, k=rows(n, kv, spread, math.copysign(1, shift)), v=(b.rows(n, kv).float() * values).to(dtype))
    return b, rows(sum(counts), heads, spread, 1)


@pytest.mark.parametrize("group", [1, 2, 3, 4])
@pytest.mark.parametrize("new,window,sinks,past", [(1024, 512, 0, 0), (1024, 512, 4, 0), (1500, 16, 0, 100), (2000, 64, 4, 0),
                                                   (2000, 512, 0, 0), (2500, 2000, 0, 0), (1100, 200, 40, 2500)])
def test_prompts_in_windows(new, window, sinks, past, group):
    """One key head, so that the keys are split over CTAs where the window allows; and with a hint that leaves them whole."""
    b, q = fill(group, [new], [past], seed=window + group)
    check(b, [new], group, window, sinks, q)
    check(b, [new], group, window, sinks, q, max_new=new, max_len=64)


@pytest.mark.parametrize("group,window,past", [(1, 2048, 4500), (2, 4096, 5000), (4, 3000, 4096)])
def test_long_windows_over_several_ctas(group, window, past):
    b, q = fill(group, [512], [past], dim=128, seed=group)
    check(b, [512], group, window, 0, q)


def test_several_heads_and_sequences():
    b, q = fill(8, [512, 300, 1], [0, 700, 40], seed=1, kv=8, block=32)
    check(b, [512, 300, 1], 8, 4096, 0, q)
    check(b, [512, 300, 1], 8, 130, 0, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("max_len", [0, 64])
@pytest.mark.parametrize("group", [1, 2, 4])
@pytest.mark.parametrize("spread,values,shift", [(1, 2.0 ** -12, 0), (1, 2.0 ** -20, 0), (1, 1e-6, 0), (1, 2.0 ** 12, 0), (4, 1, 0),
                                                 (1, 1, -20), (1, 1, -60), (1, 1, 30), (4, 2.0 ** -12, -20)])
def test_weights_far_from_one(spread, values, shift, group, max_len, dtype):
    """Small and large values, wide and shifted scores."""
    b, q = fill(group, [1024], [30], dtype=dtype, seed=group, spread=spread, values=values, shift=shift)
    for window in (100, 512):
        check(b, [1024], group, window, 0, q, max_len=max_len)
