"""The label-scoring and 8-bit cache entry points refuse bad arguments before
any device work (no GPU)."""
import ctypes

import pytest

import paper_2609_14991_gb300 as tsd
from paper_2609_14991_gb300 import _build

torch = pytest.importorskip("torch")
P = 256  # a non-NULL, aligned address; never dereferenced


@pytest.fixture(scope="module")
def L():
    _build.build()
    return tsd.lib()


def refused(L, st, word):
    assert st == tsd.TSD_EINVAL
    msg = L.tsd_last_error().decode()
    assert word in msg, msg


def test_label_scores(L):
    def call(n=2, C=10, x=P, dtype=0, ld=10, t=1.0, m=1, labels=P, k=2, logp=P, ent=P, al=P, ap=P):
        return L.tsd_label_scores(n, C, x, dtype, ld, t, m, labels, k, logp, ent, al, ap, None)

    for kw, word in [(dict(x=None), "logits"), (dict(n=(1 << 27) + 1), "n="), (dict(n=0), "n=0"), (dict(n=-1), "n=-1"), (dict(C=0), "C=0"),
                     (dict(C=262145, ld=262145), "C=262145"), (dict(dtype=3), "dtype"), (dict(ld=9), "row_stride"),
                     (dict(t=0.0), "temperature"), (dict(t=float("inf")), "temperature"), (dict(t=-1.0), "temperature"),
                     (dict(t=float("nan")), "temperature"), (dict(t=1e-45), "temperature"), (dict(m=9), "m=9"), (dict(m=-1), "m=-1"), (dict(k=9), "k=9"),
                     (dict(k=-1), "k=-1"), (dict(labels=None), "labels"), (dict(logp=None), "logp"),
                     (dict(al=None), "alt_labels"), (dict(ap=None), "alt_logp"), (dict(x=P + 2), "aligned"),
                     (dict(x=P + 1, dtype=1), "aligned")]:
        refused(L, call(**kw), word)


def test_joint_label_scores(L):
    def call(n=2, H=64, C=10, A=P, lda=64, W=P, ldw=64, t=1.0, m=0, labels=None, k=0, ws=P, nb=1 << 30):
        return L.tsd_joint_label_scores(n, H, C, A, lda, W, ldw, t, m, labels, k, P, P, P, P, ws, nb, None)

    for kw, word in [(dict(A=None), "NULL"), (dict(W=None), "NULL"), (dict(n=0), "n=0"), (dict(n=(1 << 24) + 1), "n="),
                     (dict(H=32), "H=32"), (dict(H=96), "H=96"), (dict(H=8256), "H=8256"), (dict(C=0), "C=0"),
                     (dict(C=262145), "C=262145"), (dict(lda=65), "strides"), (dict(ldw=56), "strides"),
                     (dict(A=P + 8), "aligned"), (dict(W=P + 8), "aligned"), (dict(t=0.0), "temperature"),
                     (dict(m=1), "labels"), (dict(k=9), "k=9"), (dict(n=1 << 24, C=262144), "2^40")]:
        refused(L, call(**kw), word)
    n = ctypes.c_int64()
    refused(L, L.tsd_joint_label_scores_workspace(0, 64, 10, 0, 0, ctypes.byref(n)), "n=0")
    refused(L, L.tsd_joint_label_scores_workspace(1, 64, 10, 9, 0, ctypes.byref(n)), "m=9")
    refused(L, L.tsd_joint_label_scores_workspace(1, 64, 10, 0, 0, None), "NULL")


def cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, k_tail=P, v_tail=P, dtype=1, n_blocks=4, kv_heads=2, block=16, dim=64, n_slots=3)
    d.update(kw)
    return tsd.KV8C(*d.values())


def batch(**kw):
    d = dict(n=2, slots=P, lens=P, table=P, table_width=4, starts=P, rows=5, max_new=0, max_len=0)
    d.update(kw)
    return tsd.KV8BatchC(*d.values())


def test_kv8(L):
    bad = [(dict(k=None), {}, "NULL"), (dict(v_tail=None), {}, "NULL"), (dict(k=P + 8), {}, "aligned"), (dict(dtype=0), {}, "dtype"),
           (dict(block=48), {}, "block=48"), (dict(dim=96), {}, "dim=96"), (dict(kv_heads=0), {}, "kv_heads=0"),
           (dict(n_blocks=0), {}, "n_blocks=0"), (dict(n_slots=0), {}, "n_slots=0"), ({}, dict(lens=None), "lens"),
           ({}, dict(table=None), "table"), ({}, dict(n=0), "n=0"), ({}, dict(n=65536), "n=65536"),
           ({}, dict(table_width=0), "table_width=0"), ({}, dict(table_width=1 << 27), "table_width"), ({}, dict(rows=0), "rows=0"),
           ({}, dict(rows=(1 << 22) + 1), "rows="), ({}, dict(starts=None), "starts is NULL"), ({}, dict(max_new=-1), "max_new"),
           ({}, dict(max_len=-1), "max_len")]
    nb = ctypes.c_int64()
    for c, b, word in bad:
        cc, bb = ctypes.byref(cache(**c)), ctypes.byref(batch(**b))
        refused(L, L.tsd_kv8_append(cc, bb, P, 128, 64, P, 128, 64, None), word)
        refused(L, L.tsd_kv8_read(cc, bb, P, P, None), word)
        refused(L, L.tsd_kv8_attend_workspace(cc, bb, 4, 0, 0, ctypes.byref(nb)), word)
        refused(L, L.tsd_kv8_attend(cc, bb, 4, P, 256, 64, 0.1, 0, 0, P, 256, 64, P, 0, None), word)
    c, b = ctypes.byref(cache()), ctypes.byref(batch())
    refused(L, L.tsd_kv8_append(None, b, P, 128, 64, P, 128, 64, None), "NULL")
    refused(L, L.tsd_kv8_append(c, None, P, 128, 64, P, 128, 64, None), "NULL")
    for k, row, head, word in [(None, 128, 64, "NULL k"), (P + 2, 128, 64, "aligned"), (P, 129, 64, "aligned"), (P, 128, 4, "aligned"),
                               (P, -128, 64, "out of range")]:
        refused(L, L.tsd_kv8_append(c, b, k, row, head, P, 128, 64, None), word)
    refused(L, L.tsd_kv8_read(c, b, None, P, None), "NULL")
    refused(L, L.tsd_kv8_read(c, b, P, P + 4, None), "aligned")
    for heads, window, sinks, word in [(0, 0, 0, "heads=0"), (3, 0, 0, "heads=3"), (130, 0, 0, "heads=130"), (4, -1, 0, "window"),
                                       (4, 5, -1, "sinks")]:
        refused(L, L.tsd_kv8_attend(c, b, heads, P, 256, 64, 0.1, window, sinks, P, 256, 64, P, 0, None), word)
    refused(L, L.tsd_kv8_attend(c, b, 4, None, 256, 64, 0.1, 0, 0, P, 256, 64, P, 0, None), "NULL q")
    refused(L, L.tsd_kv8_attend(c, b, 4, P, 256, 64, 0.1, 0, 0, P, 250, 64, P, 0, None), "aligned")


def test_bindings_refuse_host_tensors():
    with pytest.raises(ValueError, match="CUDA"):
        tsd.label_scores(torch.zeros(2, 3))
    with pytest.raises(ValueError, match="float32"):
        tsd.label_scores(torch.zeros(2, 3, dtype=torch.float64))
    with pytest.raises(ValueError, match="bf16"):
        tsd.joint_label_scores(torch.zeros(2, 64), torch.zeros(3, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="H = 64"):
        tsd.joint_label_scores(torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(3, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="CUDA"):
        tsd.joint_label_scores(torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(3, 64, dtype=torch.bfloat16))
    for n in (2 ** 27 + 1, 2 ** 32 + 2):  # the second would pass for 2 in 32 bits
        with pytest.raises(ValueError, match="2\\^27"):
            tsd.label_scores(torch.zeros(1, 1).expand(n, 1))
        with pytest.raises(ValueError, match="2\\^24"):
            tsd.joint_label_scores(torch.zeros(1, 64, dtype=torch.bfloat16).expand(n, 64), torch.zeros(3, 64, dtype=torch.bfloat16))
    k8, sc = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2)
    tail = torch.zeros(3, 2, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        tsd.KV8Cache(k8, k8, sc, sc, tail, tail)
    with pytest.raises(ValueError, match="k_tail"):
        tsd.KV8Cache(k8, k8, sc, sc, tail[:, :1], tail)
    with pytest.raises(ValueError, match="int8"):
        tsd.KV8Cache(k8.float(), k8, sc, sc, tail, tail)
    with pytest.raises(ValueError, match="block"):
        tsd.KV8Cache(torch.zeros(4, 2, 8, 64, dtype=torch.int8), k8, sc, sc, torch.zeros(3, 2, 2, 8, 64, dtype=torch.bfloat16), tail)


def test_temperatures_whose_exponent_factor_overflows(L):
    """log2(e) / T has to be finite too: with an infinite factor a difference of 0 would be NaN."""
    for t in (2.95e-39, 3.5e-39, 4.2e-39):
        st = L.tsd_label_scores(2, 10, P, 0, 10, t, 1, P, 2, P, P, P, P, None)
        refused(L, st, "temperature")
        refused(L, L.tsd_joint_label_scores(2, 64, 10, P, 64, P, 64, t, 0, None, 0, P, P, P, P, P, 1 << 30, None), "temperature")
