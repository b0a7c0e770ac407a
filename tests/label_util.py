"""Plain 64-bit scores of labels, for the tests of label_scores and joint_label_scores."""
import math

import torch


def oracle(x, labels, k, temperature=1.0):
    """(logp, entropy, alt_labels, alt_logp) of fp64 logits [n, C] on the CPU, row by row, from the definition."""
    n, C = x.shape
    m = 0 if labels is None else labels.shape[1]
    logp = torch.zeros(n, m, dtype=torch.float64)
    ent = torch.zeros(n, dtype=torch.float64)
    alt = torch.full((n, k), -1, dtype=torch.int32)
    altp = torch.full((n, k), -math.inf, dtype=torch.float64)
    for r in range(n):
        row = x[r]
        bad = bool(torch.isnan(row).any()) or bool((row == math.inf).any())
        y = row / temperature
        empty = bool((row == -math.inf).all())
        lse = -math.inf if empty else float(torch.logsumexp(y, 0))
        lp = torch.full_like(y, math.nan if bad else -math.inf) if bad or empty else y - lse
        p = lp.exp()
        ent[r] = math.nan if bad else 0.0 if empty else -float((p * lp)[p > 0].sum())
        for j in range(m):
            l = int(labels[r, j])
            logp[r, j] = 0.0 if l == -1 else float(lp[l]) if 0 <= l < C else math.nan
        if bad:
            altp[r] = math.nan
        else:
            order = sorted((i for i in range(C) if row[i] > -math.inf), key=lambda i: (-float(row[i]), i))[:k] if C <= 4096 \
                else [int(i) for i in torch.sort(row, descending=True, stable=True).indices[:k] if row[i] > -math.inf]
            for j, i in enumerate(order):
                alt[r, j] = i
                altp[r, j] = float(lp[i])
    return logp, ent, alt, altp


def assert_scores(got, want, what, spread):
    """Floats within the error of fp32 sums: the logarithm of a sum of up to 2^18
    terms, each with the hardware's 2^x (relative error 2^-22) of an exponent
    rounded twice (its absolute error times its weight sums to at most the
    entropy, below 13, times 2^-23), added in chains of at most 64 and a tree of
    18 (82 x 2^-24); the logit's own difference to the largest, at most `spread`,
    rounded three times: together below 8e-6 + 3 * 2^-24 * spread."""
    logp, ent, alt, altp = want
    tol = 8e-6 + 3 * 2 ** -24 * spread
    assert torch.equal(got.alt_labels.cpu(), alt), what
    for name, a, b, t in (("logp", got.logp, logp, tol), ("alt_logp", got.alt_logp, altp, tol),
                          # the entropy: the logarithm, and a mean of exponents with the same errors
                          ("entropy", got.entropy, ent, 3 * tol)):
        a = a.double().cpu().view(b.shape)
        assert torch.equal(torch.isnan(a), torch.isnan(b)), (what, name)
        assert torch.equal(torch.isinf(a), torch.isinf(b)) and torch.equal(a[torch.isinf(a)], b[torch.isinf(b)]), (what, name)
        fine = torch.isfinite(b)
        if fine.any():
            worst = float((a - b)[fine].abs().max())
            assert worst <= t, (what, name, worst, t)
