"""Residual norms on the GPU against 64 bits."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_14991_gb300 as tsd  # noqa: E402

pytestmark = pytest.mark.gpu
SUM = 2.0 ** -18  # a sum of up to 16384 terms takes at most 32 in turn and ten joins: 42 roundings of 2^-24, with the products' and root's below 2^-18
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def normed(v, e, kind, w, b, eps):
    """(result, bound) of a norm of fp64 values known within e: what e moves, and the sums', products' and
    root's own roundings."""
    if kind is None:
        return v, e
    w = torch.ones(v.shape[1], dtype=torch.float64, device=v.device) if w is None else w.double()
    b = 0.0 if b is None else b.double()
    size = v.abs().mean(1, keepdim=True)
    if kind == "layer":
        v, e = v - v.mean(1, keepdim=True), e + e.mean(1, keepdim=True) + SUM * size
    power = (v * v).mean(1, keepdim=True) + eps
    inv = power.rsqrt()
    core = v * inv * w
    moved = ((v.abs() + e) * e).mean(1, keepdim=True) / power
    return core + b, (inv * w).abs() * e + core.abs() * (moved + SUM) + 2.0 ** -23 * (core + b).abs()


def check(x, y, norm, post, gate, scale, w, b, pw, pb, eps, h, r):
    X, zero = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    if y is not None:
        z, e = normed(y.double(), zero, post, pw, pb, eps)
        f = scale * (gate.double() if gate is not None else 1.0)
        f = f * torch.ones_like(X)
        R = X + f * z
        e = f.abs() * e + 2.0 ** -22 * ((f * z).abs() + R.abs())
        tol = e + torch.finfo(r.dtype).eps / 2 * (R.abs() + e) + 2.0 ** -25
        off = (r.double() - R).abs()
        assert bool((off <= tol).all()), ("r", float((off / tol).max()))
    else:
        R, e = X, zero
        assert r is x
    if norm is None:
        assert h is None
        return
    H, e = normed(R, e, norm, w, b, eps)
    tol = e + torch.finfo(h.dtype).eps / 2 * (H.abs() + e) + 2.0 ** -25
    off = (h.double() - H).abs()
    assert bool((off <= tol).all()), ("h", float((off / tol).max()))


def make(n, d, dtype, x_dtype, gate=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = (2 * rand(n, d) + 0.5).to(x_dtype).cuda()
    y = (0.7 * rand(n, d) - 0.2).to(dtype).cuda()
    v = [(1 + 0.3 * rand(d)).cuda(), (0.1 * rand(d)).cuda(), (1 + 0.3 * rand(d)).cuda(), (0.1 * rand(d)).cuda()]
    gt = None if gate is None else torch.tanh(rand(*((n, d) if gate == "rows" else (d,)))).to(dtype).cuda()
    return x, y, v, gt


TYPES = [(BF, BF), (BF, FL), (HF, HF), (HF, FL), (FL, FL)]


@pytest.mark.parametrize("dtype,x_dtype", TYPES)
@pytest.mark.parametrize("norm,post", [("rms", None), ("layer", None), ("rms", "rms"), ("layer", "layer"), ("rms", "layer"), (None, "rms"), (None, None)])
@pytest.mark.parametrize("gate", [None, "channels", "rows"])
def test_kinds_and_types(dtype, x_dtype, norm, post, gate):
    for d in (64, 96, 77):
        x, y, (w, b, pw, pb), gt = make(5, d, dtype, x_dtype, gate)
        kw = dict(norm=norm, weight=w if norm else None, bias=b if norm == "layer" else None, post=post,
                  post_weight=pw if post else None, post_bias=pb if post == "layer" else None)
        h, r = tsd.residual_norm(x, y, gate=gt, scale=0.5, **kw)
        check(x, y, norm, post, gt, 0.5, kw["weight"], kw["bias"], kw["post_weight"], kw["post_bias"], 1e-5, h, r)


@pytest.mark.parametrize("d", [1, 2, 7, 8, 31, 255, 256, 257, 512, 520, 1023, 1024, 1025, 1032, 2047, 2048, 2056, 4096, 4104, 5000, 8191, 8192, 8200,
                               16383, 16384])
@pytest.mark.parametrize("dtype,x_dtype", [(BF, BF), (HF, FL)])
def test_widths(d, dtype, x_dtype):
    x, y, (w, b, pw, pb), gt = make(3, d, dtype, x_dtype, "rows", seed=d)
    h, r = tsd.residual_norm(x, y, norm="layer", weight=w, bias=b, post="layer", post_weight=pw, post_bias=pb, gate=gt, scale=0.7)
    check(x, y, "layer", "layer", gt, 0.7, w, b, pw, pb, 1e-5, h, r)
    h, r = tsd.residual_norm(x, y, norm="rms", post="rms", eps=1e-6)
    check(x, y, "rms", "rms", None, 1.0, None, None, None, None, 1e-6, h, r)


@pytest.mark.parametrize("d", [1, 7, 8, 33, 64, 65, 128, 129, 256, 257, 505, 512, 513, 1017, 1024, 1025, 2041, 2048, 2049, 4089, 4097, 8192, 8193, 16376, 16378, 16384])
@pytest.mark.parametrize("dtype,x_dtype", [(HF, HF), (BF, FL)])
def test_widths_of_many_rows(d, dtype, x_dtype):
    """Enough rows for as few threads per row as any number takes; odd widths, whose rows stand off multiples of eight elements."""
    x, y, (w, b, pw, pb), gt = make(1003, d, dtype, x_dtype, "rows" if d % 2 else "channels", seed=d)
    h, r = tsd.residual_norm(x, y, norm="layer", weight=w, bias=b, post="rms", post_weight=pw, gate=gt, scale=0.7)
    check(x, y, "layer", "rms", gt, 0.7, w, b, pw, None, 1e-5, h, r)
    h, r = tsd.residual_norm(x, y, norm="rms", post="layer", post_weight=pw, post_bias=pb)
    check(x, y, "rms", "layer", None, 1.0, None, None, pw, pb, 1e-5, h, r)


@pytest.mark.parametrize("n,d", [(40001, 33), (40001, 64), (20011, 200), (20001, 500), (9001, 1000), (9001, 1024), (5003, 1537), (5003, 2048), (3001, 4001), (1999, 6001)])
@pytest.mark.parametrize("dtype,x_dtype", [(BF, BF), (HF, FL)])
def test_many_rows(n, d, dtype, x_dtype):
    """More rows than the device holds at once, an odd number of them; in place with the same bits."""
    x, y, (w, b, pw, _), gt = make(n, d, dtype, x_dtype, "rows", seed=n)
    h, r = tsd.residual_norm(x, y, norm="layer", weight=w, bias=b, post="rms", post_weight=pw, gate=gt)
    check(x, y, "layer", "rms", gt, 1.0, w, b, pw, None, 1e-5, h, r)
    tsd.residual_norm(x, y, norm="layer", weight=w, bias=b, post="rms", post_weight=pw, gate=gt, out=(y, x))
    assert torch.equal(x, r) and torch.equal(y, h)


@pytest.mark.parametrize("d", [40, 333, 3000, 9000])
@pytest.mark.parametrize("n", [3, 2000])
def test_arrays_that_stand_apart(d, n):
    """Row arrays each off by another number of elements, and with other distances of rows."""
    x, y, (w, b, pw, _), gt = make(n, d, BF, FL, "rows", seed=d)
    def apart(t, shift, pad):  # noqa: E306
        v = torch.full((n * (d + pad) + 16,), 9.0, dtype=t.dtype, device="cuda")[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
        v.copy_(t)
        return v
    h, r = apart(y, 5, 7), apart(x, 2, 1)
    tsd.residual_norm(apart(x, 1, 3), apart(y, 3, 0), norm="layer", weight=w, bias=b, post="rms", post_weight=pw, gate=apart(gt, 0, 2), scale=0.3, out=(h, r))
    check(x, y, "layer", "rms", gt, 0.3, w, b, pw, None, 1e-5, h, r)
    # ... and alike, but off a multiple of eight
    h, r = apart(y, 3, 5), apart(x, 3, 5)
    tsd.residual_norm(apart(x, 3, 5), apart(y, 3, 5), norm="layer", weight=w, bias=b, gate=apart(gt, 3, 5), out=(h, r))
    check(x, y, "layer", None, gt, 1.0, w, b, None, None, 1e-5, h, r)


@pytest.mark.parametrize("shift", [1, 4])
def test_weights_at_any_float(shift):
    x, y, (w, b, _, _), gt = make(1200, 512, BF, BF, "channels", seed=2)
    w2, b2 = (torch.cat([torch.zeros(shift, device="cuda"), t])[shift:] for t in (w, b))
    g2 = torch.cat([torch.zeros(shift, dtype=BF, device="cuda"), gt])[shift:]
    for n in (3, 1200):
        h, r = tsd.residual_norm(x[:n], y[:n], norm="layer", weight=w2, bias=b2, gate=g2)
        check(x[:n], y[:n], "layer", None, gt, 1.0, w, b, None, None, 1e-5, h, r)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 127, 1000])
@pytest.mark.parametrize("d", [64, 512, 1536])
def test_rows(n, d):
    x, y, (w, b, _, _), _ = make(n, d, BF, FL, seed=n)
    h, r = tsd.residual_norm(x, y, norm="layer", weight=w, bias=b, scale=0.5)
    check(x, y, "layer", None, None, 0.5, w, b, None, None, 1e-5, h, r)
    one = [tsd.residual_norm(x[i:i + 1], y[i:i + 1], norm="layer", weight=w, bias=b, scale=0.5) for i in (0, n - 1)]
    for i, (a, c) in zip((0, n - 1), one):  # a row's bits do not depend on the others
        assert torch.equal(a[0], h[i]) and torch.equal(c[0], r[i])


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_a_norm_alone(dtype, norm):
    for d in (40, 511):
        x, _, (w, b, _, _), _ = make(6, d, dtype, dtype)
        h, r = tsd.residual_norm(x, norm=norm, weight=w, bias=b)
        check(x, None, norm, None, None, 1.0, w, b, None, None, 1e-5, h, r)


@pytest.mark.parametrize("shift,pad", [(0, 0), (0, 8), (1, 0), (0, 3), (8, 16)])
def test_strides_and_alignment(shift, pad):
    n, d = 6, 128
    def inside(t):  # noqa: E306
        buf = torch.full((n * (d + pad) + 16,), 9.0, dtype=t.dtype, device="cuda")
        v = buf[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
        v.copy_(t)
        return buf, v
    x, y, (w, b, pw, pb), gt = make(n, d, BF, FL, "rows")
    (_, xs), (_, ys), (_, gs) = inside(x), inside(y), inside(gt)
    (hb, h), (rb, r) = inside(torch.zeros(n, d, dtype=BF, device="cuda")), inside(torch.zeros(n, d, device="cuda"))
    a, c = tsd.residual_norm(xs, ys, norm="rms", weight=w, post="rms", post_weight=pw, gate=gs, scale=0.3, out=(h, r))
    assert a is h and c is r
    check(x, y, "rms", "rms", gt, 0.3, w, None, pw, None, 1e-5, h, r)
    assert int((hb == 9).sum()) >= hb.numel() - n * d and int((rb == 9).sum()) >= rb.numel() - n * d  # nothing between the rows


@pytest.mark.parametrize("d", [64, 1000, 4096, 333])
def test_in_place(d):
    x, y, (w, _, pw, _), _ = make(9, d, BF, BF)
    h, r = tsd.residual_norm(x, y, weight=w, post="rms", post_weight=pw)
    x2, y2 = x.clone(), y.clone()
    tsd.residual_norm(x2, y2, weight=w, post="rms", post_weight=pw, out=(y2, x2))
    assert torch.equal(x2, r) and torch.equal(y2, h)


def test_a_broadcast_gate_row_and_an_expanded_stream():
    x, y, (w, _, _, _), gt = make(7, 48, HF, FL, "channels")
    a = tsd.residual_norm(x, y, weight=w, gate=gt)
    b = tsd.residual_norm(x, y, weight=w, gate=gt[None].repeat(7, 1))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    with pytest.raises(ValueError, match="overlap"):
        tsd.residual_norm(x[:1].expand(7, 48), y, weight=w)


def test_values_at_the_ends():
    """Zero rows, infinities and NaN reach the results of their rows alone, as the formula has them."""
    x, y, (w, b, pw, pb), _ = make(6, 72, BF, FL)
    x[0], y[0] = 0, 0
    x[1, 5] = float("inf")
    y[2, 71] = float("nan")
    x[3], y[3] = 1e15, 0
    x[4], y[4] = 3.0, 0  # a constant row: its layer norm is the bias
    for norm in ("rms", "layer"):
        h, r = tsd.residual_norm(x, y, norm=norm, weight=w, bias=b)
        want_r = x.double() + y.double()
        v = want_r - (want_r.mean(1, keepdim=True) if norm == "layer" else 0)
        want = v / ((v * v).mean(1, keepdim=True) + 1e-5).sqrt() * w.double() + b.double()
        for i in (1, 2):
            assert torch.equal(torch.isnan(h[i]), torch.isnan(want[i])), (norm, i)
            assert torch.equal(torch.isnan(r[i]), torch.isnan(want_r[i]))
        rows = [0, 5] if norm == "layer" else [0, 3, 4, 5]
        tol = 2.0 ** -8 * want.abs() + SUM * 8 + 2.0 ** -25
        assert bool(((h.double() - want).abs() <= tol)[rows].all())
        if norm == "layer":  # deviations of a constant: those of its sum, 42 roundings of 2^-24 of it, over sqrt(eps)
            assert bool(((h[4].double() - b.double()).abs() <= 2.0 ** -8 * b.double().abs() + 42 * 2.0 ** -24 * 3 / 1e-5 ** 0.5 * w.double().abs()).all())


def test_zero_eps():
    x = torch.zeros(2, 16, device="cuda")
    x[1] = 2
    h, _ = tsd.residual_norm(x, norm="rms", eps=0.0)
    assert bool(torch.isnan(h[0]).all()) and bool((h[1] == 1).all())


def test_a_replayed_graph_and_another_stream():
    x, y, (w, _, _, _), _ = make(4, 256, BF, BF)
    h, r = torch.empty_like(x), torch.empty_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tsd.residual_norm(x, y, weight=w, out=(h, r))
    for i in range(2):
        y.copy_(make(4, 256, BF, BF, seed=i + 5)[1])
        g.replay()
        check(x, y, "rms", None, None, 1.0, w, None, None, None, 1e-5, h, r)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    a, c = tsd.residual_norm(x, y, weight=w, stream=s)
    s.synchronize()
    assert torch.equal(a, h) and torch.equal(c, r)


def test_binding_refusals():
    x, y, (w, b, _, _), gt = make(4, 64, BF, FL, "rows")
    for kw, word in [(dict(x=x, y=y[:3]), "y must"), (dict(x=x, y=y, weight=w[:3]), "weights"), (dict(x=x, y=y, weight=w.half()), "weights"),
                     (dict(x=x, y=y, gate=gt.float()), "gate"), (dict(x=x, y=y, gate=gt[:2]), "gate"), (dict(x=x, gate=gt), "without y"),
                     (dict(x=x, post="rms"), "without y"), (dict(x=x, norm=None), "without y"), (dict(x=x, y=y, norm=None, weight=w), "has a weight"),
                     (dict(x=x, y=y, out=(x, x)), "out's h"), (dict(x=x, y=y, out=(None, y)), "out's r"), (dict(x=x.t(), y=y.t()), "adjacent"),
                     (dict(x=x, y=y, gate=gt[0, ::2].repeat(2)[:64].cpu()), "gate"), (dict(x=x, y=y.cpu()), "y must")]:
        with pytest.raises(ValueError, match=word):
            tsd.residual_norm(**kw)
    with pytest.raises(tsd.TsdError, match="eps"):
        tsd.residual_norm(x, y, eps=-1.0)
    with pytest.raises(tsd.TsdError, match="scale"):
        tsd.residual_norm(x, y, scale=float("inf"))


@pytest.mark.parametrize("d", [64, 200, 264, 512, 520, 1000, 1024, 1536, 2048, 4096, 5000, 8184, 8192, 12000])
@pytest.mark.parametrize("norm,post", [("rms", "layer"), ("layer", "rms")])
def test_bits_do_not_depend_on_other_rows(d, norm, post):
    """Rows alone, in calls of some and of more than the device holds at once: in fp32, after a norm on both sides, bit by bit."""
    n = 1200
    x, y, (w, b, pw, pb), gt = make(n, d, FL, FL, "channels", seed=d)
    kw = dict(norm=norm, weight=w, bias=b, post=post, post_weight=pw, post_bias=pb if post == "layer" else None, gate=gt, scale=0.7)
    h, r = tsd.residual_norm(x, y, **kw)
    for a, c in [(0, 1), (1199, 1200), (500, 503), (100, 300), (0, 900), (250, 1199)]:
        h2, r2 = tsd.residual_norm(x[a:c], y[a:c], **kw)
        assert torch.equal(h2, h[a:c]) and torch.equal(r2, r[a:c]), (a, c)


@pytest.mark.parametrize("d", [63, 249, 257, 505, 777, 1017, 1021, 2043, 4095, 8191])
def test_bits_of_odd_widths_do_not_depend_on_other_rows(d):
    """The same of rows that stand off multiples of eight elements, where all arrays of the calls stand alike."""
    n = 1200
    x, y, (w, b, pw, _), gt = make(n, d, FL, FL, "rows", seed=d)
    kw = dict(norm="layer", weight=w, bias=b, post="rms", post_weight=pw)
    h, r = tsd.residual_norm(x, y, gate=gt, **kw)
    for a, c in [(0, 1), (7, 8), (8, 9), (1199, 1200), (500, 503), (100, 300), (251, 1199)]:
        h2, r2 = torch.zeros_like(h), torch.zeros_like(r)
        tsd.residual_norm(x[a:c], y[a:c], gate=gt[a:c], out=(h2[a:c], r2[a:c]), **kw)
        assert torch.equal(h2[a:c], h[a:c]) and torch.equal(r2[a:c], r[a:c]), (a, c)


def test_results_that_a_call_does_not_write_are_refused():
    x, y, (w, _, _, _), _ = make(4, 64, BF, BF)
    h, r = torch.zeros_like(x), torch.zeros_like(x)
    with pytest.raises(ValueError, match="no h to write"):
        tsd.residual_norm(x, y, norm=None, out=(h, r))
    with pytest.raises(ValueError, match="no r to write"):
        tsd.residual_norm(x, weight=w, out=(h, r))
    a, b = tsd.residual_norm(x, weight=w, out=(h, x))
    assert a is h and b is x
    check(x, None, "rms", None, None, 1.0, w, None, None, None, 1e-5, h, x)
    a, b = tsd.residual_norm(x, y, norm=None, out=(None, r))
    assert a is None and b is r
    check(x, y, None, None, None, 1.0, None, None, None, None, 1e-5, None, r)


@pytest.mark.parametrize("pad", [64, 65])
@pytest.mark.parametrize("d", [512, 333])
def test_far_rows(d, pad):
    """Rows whose offsets pass 2^32 elements, in whole groups of eight, off them, and (the gate) apart from the others."""
    far = 2 ** 31 + pad
    buf = torch.empty(3 * far, dtype=BF, device="cuda")
    x, y, h, r, gt = (buf[1024 * i:].as_strided((3, d), (far, 1)) for i in range(5))
    a, b, (w, _, pw, _), c = make(3, d, BF, BF, "rows", seed=d)
    x.copy_(a), y.copy_(b), gt.copy_(c)
    tsd.residual_norm(x, y, weight=w, post="layer", post_weight=pw, gate=gt, out=(h, r))
    check(a, b, "rms", "layer", c, 1.0, w, None, pw, None, 1e-5, h, r)
    tsd.residual_norm(x, y, weight=w, post="layer", post_weight=pw, gate=c, out=(y, x))
    check(a, b, "rms", "layer", c, 1.0, w, None, pw, None, 1e-5, y, x)
