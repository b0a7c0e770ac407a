"""Rotary positions, residual norms and attention over encoder states refuse bad
arguments before any device work, and the host's frequencies are the formula's (no GPU)."""
import concurrent.futures
import ctypes
import math
import threading
from decimal import Decimal, getcontext

import numpy as np
import pytest

import paper_2609_14991_gb300 as tsd
from paper_2609_14991_gb300 import _build

torch = pytest.importorskip("torch")
P = 256  # a non-NULL, aligned address; never dereferenced
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def L():
    _build.build()
    return tsd.lib()


def refused(L, st, word):
    assert st == tsd.TSD_EINVAL
    msg = L.tsd_last_error().decode()
    assert word in msg, msg


def cfg(rot=64, scaling=0, base=10000.0, factor=8.0, original=4096.0, low=1.0, high=32.0):
    return tsd.RotaryCfgC(rot, scaling, base, factor, original, low, high)


def turns_of(L, c):
    t = np.zeros(c.rot // 2, dtype=np.uint64)
    assert L.tsd_rotary_turns(ctypes.byref(c), t.ctypes.data) == 0, L.tsd_last_error()
    return t


def frequency(c, i):
    half = c.rot // 2
    base = c.base * (c.factor ** (half / (half - 1)) if c.scaling == 2 and half > 1 else 1)
    f = base ** (-i / half)
    if c.scaling == 1:
        f /= c.factor
    if c.scaling == 3:
        keep = min(1.0, max(0.0, (c.original * f / (2 * math.pi) - c.low) / (c.high - c.low)))
        f = f * keep + f / c.factor * (1 - keep)
    return f


@pytest.mark.parametrize("rot", [2, 4, 64, 128, 1024])
@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 0.5])
def test_turns(L, rot, scaling, base):
    """Fractions of a turn, mod 2^64: the power is good to a few units of 2^-53 of itself (2^-49 is
    allowed), the rest to two units."""
    getcontext().prec = 60
    c = cfg(rot, scaling, base)
    for i, t in enumerate(turns_of(L, c)):
        f = frequency(c, i)
        want = (Decimal(f) / (2 * PI)) * 2 ** 64 % 2 ** 64
        off = abs((Decimal(int(t)) - want + 2 ** 63) % 2 ** 64 - 2 ** 63)
        assert off <= Decimal(f) / 6 * 2 ** 15 + 2, (i, f, off)


def test_turns_refusals(L):
    t = np.zeros(512, dtype=np.uint64)
    for kw, word in [(dict(rot=0), "rot=0"), (dict(rot=3), "rot=3"), (dict(rot=1026), "rot=1026"), (dict(base=0.0), "base"),
                     (dict(base=-1.0), "base"), (dict(base=math.inf), "base"), (dict(base=math.nan), "base"), (dict(scaling=4), "scaling"),
                     (dict(scaling=-1), "scaling"), (dict(scaling=1, factor=0.0), "factor"), (dict(scaling=2, factor=math.inf), "factor"),
                     (dict(scaling=3, original=0.0), "ramp"), (dict(scaling=3, low=2.0, high=2.0), "ramp"),
                     (dict(scaling=3, high=math.nan), "ramp"), (dict(base=1e-300), "2^52"), (dict(scaling=1, factor=1e-300), "2^52")]:
        refused(L, L.tsd_rotary_turns(ctypes.byref(cfg(**kw)), t.ctypes.data), word)
    refused(L, L.tsd_rotary_turns(None, t.ctypes.data), "NULL")
    refused(L, L.tsd_rotary_turns(ctypes.byref(cfg()), None), "NULL")


def test_rotary_refusals(L):
    def call(rot=(), rows=(), q=(), k=(), with_k=True):
        r = dict(turns=P, dim=64, rot=64, interleaved=0, dtype=1, magnitude=1.0)
        w = dict(rows=3, positions=None, n=2, slots=P, lens=P, starts=P, n_slots=4)
        h = dict(x=P, out=P, row=512, head=64, out_row=512, out_head=64, heads=8)
        h2 = {**h, "x": 2 * P, "out": 2 * P}
        a, b = tsd.RotaryC(*{**r, **dict(rot)}.values()), tsd.RotaryRowsC(*{**w, **dict(rows)}.values())
        c, d = tsd.RotaryHeadsC(*{**h, **dict(q)}.values()), tsd.RotaryHeadsC(*{**h2, **dict(k)}.values())
        return L.tsd_rotary_apply(ctypes.byref(a), ctypes.byref(b), ctypes.byref(c), ctypes.byref(d) if with_k else None, None)

    for kw, word in [(dict(turns=None), "turns"), (dict(turns=P + 4), "turns"), (dict(dim=1), "dim=1"), (dict(dim=1026), "dim=1026"),
                     (dict(rot=66), "rot=66"), (dict(rot=0), "rot=0"), (dict(rot=7), "rot=7"), (dict(dtype=3), "dtype"),
                     (dict(magnitude=math.inf), "magnitude"), (dict(magnitude=math.nan), "magnitude")]:
        refused(L, call(rot=kw.items()), word)
    for kw, word in [(dict(rows=0), "rows=0"), (dict(rows=(1 << 22) + 1), "rows="), (dict(positions=P), "positions, or"),
                     (dict(lens=None), "NULL positions"), (dict(n=0), "n=0"), (dict(n=65536), "n=65536"), (dict(n_slots=0), "n_slots=0"),
                     (dict(starts=None), "starts is NULL")]:
        refused(L, call(rows=kw.items()), word)
    for kw, word in [(dict(x=None), "NULL"), (dict(out=None), "NULL"), (dict(heads=0), "heads=0"), (dict(heads=1025), "heads=1025"),
                     (dict(x=P + 1), "aligned"), (dict(row=-1), "strides"), (dict(out_head=1 << 41), "strides"),
                     (dict(out_row=63), "overlap"), (dict(out_head=0), "overlap"), (dict(row=1024), "in place"), (dict(head=72), "in place")]:
        refused(L, call(q=kw.items()), word)
        refused(L, call(k=kw.items()), word)
    refused(L, call(q=dict(out=2 * P).items()), "queries and keys overlap")
    refused(L, call(k=dict(out=P).items()), "queries and keys overlap")
    refused(L, L.tsd_rotary_apply(None, None, None, None, None), "NULL")


def test_residual_norm_refusals(L):
    norm = lambda **kw: ctypes.byref(tsd.NormC(*{**dict(kind=1, eps=1e-5, weight=P, bias=None), **kw}.values()))  # noqa: E731

    def call(n=3, d=16, x=P, xt=1, xr=16, y=2 * P, yt=1, yr=16, post=None, gate=None, gr=0, scale=1.0, nm=norm(), r=P, rr=16, h=2 * P, hr=16):
        return L.tsd_residual_norm(n, d, x, xt, xr, y, yt, yr, post, gate, gr, scale, nm, r, rr, h, hr, None)

    for kw, word in [(dict(n=0), "n=0"), (dict(n=(1 << 27) + 1), "n="), (dict(d=0), "d=0"), (dict(d=16385, xr=16385), "d=16385"),
                     (dict(yt=3), "dtype"), (dict(yt=-1), "dtype"), (dict(xt=2), "dtype"), (dict(yt=0), "dtype"), (dict(x=None), "NULL x"),
                     (dict(x=P + 1), "aligned"), (dict(xr=15), "x overlap"), (dict(yr=15), "y overlap"), (dict(r=None), "NULL r"),
                     (dict(h=None), "NULL h"), (dict(hr=15), "h overlap"), (dict(gate=P, gr=15), "gate overlap"), (dict(gate=P + 1), "gate"),
                     (dict(scale=math.inf), "scale"), (dict(scale=math.nan), "scale"), (dict(nm=norm(kind=3)), "kind 3"),
                     (dict(post=norm(kind=-1)), "kind -1"), (dict(nm=norm(eps=-1.0)), "eps"), (dict(post=norm(eps=math.nan)), "eps"),
                     (dict(nm=norm(weight=P + 2)), "weight"), (dict(y=None, gate=P), "without y"), (dict(y=None, post=norm()), "without y"),
                     (dict(y=None, nm=None), "without y"), (dict(h=P), "overlap"), (dict(r=2 * P), "overlap"), (dict(r=3 * P, h=P), "overlap"),
                     (dict(xr=32), "overlap"), (dict(yr=32), "overlap"), (dict(y=None, xr=32, h=P), "overlap"), (dict(r=3 * P, h=3 * P), "overlap")]:
        refused(L, call(**kw), word)


def test_residual_norm_refuses_results_over_what_other_rows_read(L):
    """A gate, weights or biases in the memory of r or h: rows would race for them."""
    F = 1 << 20
    norm = lambda **kw: ctypes.byref(tsd.NormC(*{**dict(kind=1, eps=1e-5, weight=F, bias=None), **kw}.values()))  # noqa: E731

    def call(n=3, d=16, x=P, xr=40, y=4096, yr=40, post=None, gate=None, gr=0, nm=norm(), r=8192, rr=40, h=16384, hr=40, xt=1):
        return L.tsd_residual_norm(n, d, x, xt, xr, y, 1, yr, post, gate, gr, 1.0, nm, r, rr, h, hr, None)

    for gr in (0, 40):
        refused(L, call(gate=8192, gr=gr), "gate")
        refused(L, call(gate=16384, gr=gr), "gate")
        refused(L, call(gate=P, gr=gr, r=P), "gate")     # x in place, and the gate is x
        refused(L, call(gate=4096, gr=gr, h=4096), "gate")  # likewise y
    for at, word in [(8192 + 30, "gate"), (8192 - 30, "gate"), (8192 + 2 * 80, "gate"), (16384 + 80 + 30, "gate"), (16384 + 2 * 80 - 2, "gate")]:
        refused(L, call(gate=at), word)
    for at in (8192, 8192 - 60, 8192 + 28, 8192 + 2 * 80 + 28, 16384, 16384 + 80):
        refused(L, call(nm=norm(weight=at)), "weight")
        refused(L, call(nm=norm(bias=at)), "bias")
        refused(L, call(post=norm(weight=at)), "weight")
        refused(L, call(post=norm(bias=at)), "bias")
    refused(L, call(y=None, nm=norm(weight=16384 + 4)), "weight")


def test_cross_refusals(L):
    def call(s=(), b=(), heads=4, q=P, qr=256, qh=64, scale=0.1, out=P, orow=256, oh=64, ws=None, nws=0):
        x = dict(k=P, v=P, ks=4096, kf=128, kh=64, vs=4096, vf=128, vh=64, lens=P, dtype=1, n_sources=3, frames=32, kv_heads=2, dim=64)
        w = dict(n=2, sources=P, starts=P, rows=5, max_rows=0)
        x, w = tsd.StatesC(*{**x, **dict(s)}.values()), tsd.CrossBatchC(*{**w, **dict(b)}.values())
        return L.tsd_cross_attend(ctypes.byref(x), ctypes.byref(w), heads, q, qr, qh, scale, out, orow, oh, ws, nws, None)

    for kw, word in [(dict(k=None), "NULL k"), (dict(v=None), "NULL v"), (dict(k=P + 8), "aligned"), (dict(kf=127), "aligned"), (dict(vh=4), "aligned"),
                     (dict(ks=-4096), "range"), (dict(vs=1 << 37), "range"), (dict(dtype=0), "dtype"), (dict(dim=96), "dim=96"),
                     (dict(kv_heads=0), "kv_heads=0"), (dict(n_sources=0), "n_sources=0"), (dict(frames=0), "frames=0"),
                     (dict(frames=(1 << 30) + 1), "frames=")]:
        refused(L, call(s=kw.items()), word)
    for kw, word in [(dict(n=0), "n=0"), (dict(n=65536), "n=65536"), (dict(rows=0), "rows=0"), (dict(rows=(1 << 22) + 1), "rows="),
                     (dict(starts=None), "starts is NULL"), (dict(n=4, sources=None), "sources is NULL"), (dict(max_rows=-1), "max_rows")]:
        refused(L, call(b=kw.items()), word)
    for kw, word in [(dict(heads=0), "heads=0"), (dict(heads=3), "heads=3"), (dict(heads=130), "heads=130"), (dict(q=None), "NULL q"),
                     (dict(out=None), "NULL out"), (dict(qr=250), "aligned"), (dict(out=P + 2), "aligned"), (dict(oh=-64), "range"),
                     (dict(scale=math.inf), "scale"), (dict(scale=math.nan), "scale"), (dict(orow=56), "overlap"), (dict(oh=0), "overlap")]:
        refused(L, call(**kw), word)
    refused(L, L.tsd_cross_attend(None, None, 4, P, 256, 64, 0.1, P, 256, 64, None, 0, None), "NULL")
    need = ctypes.c_int64()
    refused(L, L.tsd_cross_attend_workspace(None, None, 4, ctypes.byref(need)), "NULL")
    refused(L, L.tsd_cross_attend_workspace(None, None, 4, None), "NULL")


def test_bindings_refuse():
    bf = torch.bfloat16
    with pytest.raises(ValueError, match="rot"):
        tsd.Rotary(64, 66, device="cpu")
    with pytest.raises(ValueError, match="layout"):
        tsd.Rotary(64, layout="other", device="cpu")
    with pytest.raises(ValueError, match="scaling"):
        tsd.Rotary(64, scaling="other", device="cpu")
    with pytest.raises(tsd.TsdError, match="factor"):
        tsd.Rotary(64, scaling="linear", factor=0.0, device="cpu")
    x = torch.zeros(2, 16, dtype=bf)
    for kw, word in [(dict(x=x.view(-1)), "n, d"), (dict(x=x, norm="other"), "norms are"), (dict(x=x.double()), "float32"), (dict(x=x, y=x.half()), "same type"),
                     (dict(x=x), "CUDA"), (dict(x=torch.zeros(1, 16385)), "16384"), (dict(x=torch.zeros(1, 1).expand(2 ** 27 + 1, 1)), "2\\^27")]:
        with pytest.raises(ValueError, match=word):
            tsd.residual_norm(**kw)
    k = torch.zeros(2, 5, 1, 64, dtype=bf)
    for a, word in [((k.float(), k), "bf16"), ((k, k[:1]), "v must"), ((k, k.half()), "v must"), ((k[..., :32], k[..., :32]), "dim is"), ((k, k), "CUDA")]:
        with pytest.raises(ValueError, match=word):
            tsd.CrossStates(*a)


def test_a_first_call_beside_another_threads_first_call(monkeypatch):
    """What the bindings keep of torch is complete before a thread can find it (torch's calls are replaced: no GPU)."""
    inside, done, first = threading.Event(), threading.Event(), threading.Lock()

    def device_count():
        if first.acquire(blocking=False):  # the thread that came first waits here until the other's call has ended
            inside.set()
            done.wait(5)
        return 2

    for name in ("_new_empty", "_get_device", "_get_raw_stream", "_F32", "_I32", "_U8"):
        monkeypatch.setattr(tsd, name, None)
    monkeypatch.setattr(tsd, "_devices", {})
    monkeypatch.setattr(torch.cuda, "init", lambda: None)
    monkeypatch.setattr(torch.cuda, "device_count", device_count)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 7 + dev, raising=False)
    monkeypatch.setattr(torch, "empty", lambda n, dtype, device: (n, dtype, device))

    def calls():
        return tsd._current_device(), tsd._empty(3, torch.float32, 1, None), tsd._workspace(5, 0, None), tsd._raw_stream(None, 1)

    with concurrent.futures.ThreadPoolExecutor(2) as ex:
        a = ex.submit(calls)
        assert inside.wait(5)
        b = ex.submit(calls)
        try:
            got = b.result(5)
        finally:
            done.set()
        assert got == a.result(5) == (1, (3, torch.float32, torch.device("cuda", 1)), (5, torch.uint8, torch.device("cuda", 0)), 8)
