"""A decoder's layer as a program runs it: positions turned into queries and keys, the
cache's append and attention, a norm around it, attention over an encoder's states, the
next norm; each step against 64 bits on what it was given, and the whole captured."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_14991_gb300 as tsd  # noqa: E402
from tests import test_gpu_cross_attend as cross  # noqa: E402
from tests import test_gpu_residual_norm as norms  # noqa: E402
from tests import test_gpu_rotary as rotary  # noqa: E402
from tests.kv8_util import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def weights(d, seed):
    g = torch.Generator().manual_seed(seed)
    return [(s + 0.2 * torch.randn(d, generator=g)).cuda() for s in (1.0, 0.0, 1.0)]


@pytest.mark.parametrize("dim,heads,kv,layout", [(64, 4, 2, "half"), (128, 2, 2, "interleaved")])
def test_prompts_and_tokens(dim, heads, kv, layout):
    calls = [[20, 7, 33], [1, 1, 1], [3, 0, 2], [70, 1, 4]]
    total = [sum(c[i] for c in calls) for i in range(3)]
    b = Batch(tsd, total, kv, 16, dim, seed=dim)
    turn = tsd.Rotary(dim, layout=layout)
    frames, sources = [150, 0, 41], [2, 0, 0]  # the second and third sequences read one source, of 150 frames
    k, v = cross.make(3, 160, kv, dim, seed=3)
    states = tsd.CrossStates(k, v, cross.ints(frames))
    d = heads * dim
    w, bias, pw = weights(d, dim)
    for step, counts in enumerate(calls):
        rows = sum(counts)
        qkv = rotary.rand(rows, heads + 2 * kv, dim, seed=step)
        q, new, values = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        pos = [b.len[i] + t for i, c in enumerate(counts) for t in range(c)]
        b.len = [x + c for x, c in zip(b.len, counts)]
        a = b.args(counts)
        b.len = [x - c for x, c in zip(b.len, counts)]
        tq, tk = turn(q, new, lens=a["lens"], starts=a["starts"], slots=a["slots"])
        rotary.check(tq, q, pos, dim, layout)
        rotary.check(tk, new, pos, dim, layout)
        b.append(counts, k=tk, v=values)
        y = b.check_attend(counts, heads, q=tq)
        x = torch.randn(rows, d, generator=torch.Generator().manual_seed(step + 9)).cuda()
        h, r = tsd.residual_norm(x, y.view(rows, d), norm="rms", weight=w, post="rms", post_weight=pw)
        norms.check(x, y.view(rows, d), "rms", "rms", None, 1.0, w, None, pw, None, 1e-5, h, r)
        q2 = h.view(rows, heads, dim)
        y2 = states.attend(q2, starts=a["starts"], sources=cross.ints(sources), max_rows=max(counts))
        cross.check(y2, k, v, frames, q2, counts, sources)
        h2, r2 = tsd.residual_norm(r, y2.view(rows, d), norm="layer", weight=w, bias=bias, scale=0.5, out=(None, r))
        assert r2 is r  # in place: checked below from a copy
        keep = torch.empty_like(r)
        h3, _ = tsd.residual_norm(tsd.residual_norm(x, y.view(rows, d), norm=None, post="rms", post_weight=pw)[1], y2.view(rows, d), norm="layer",
                                  weight=w, bias=bias, scale=0.5, out=(None, keep))
        assert torch.equal(h2, h3) and torch.equal(r, keep)
    b.check_held()


def test_captured_tokens():
    """Single tokens of three sequences, a layer per replay: lengths grow in the graph; the same bits as without."""
    dim, heads, kv, n = 64, 4, 2, 3
    d = heads * dim
    turn = tsd.Rotary(dim)
    w, bias, _ = weights(d, 1)
    k, v = cross.make(n, 90, kv, dim, seed=4)
    states = tsd.CrossStates(k, v, cross.ints([90, 13, 50]))
    qkv = torch.zeros(n, heads + 2 * kv, dim, dtype=BF, device="cuda")
    x = torch.zeros(n, d, device="cuda")
    table = torch.randperm(24, generator=torch.Generator().manual_seed(2)).int().view(n, 8).cuda()

    def layer(cache, lens, x):
        lens += 1
        q, new = turn(qkv[:, :heads], qkv[:, heads:heads + kv], lens=lens)
        cache.append(new, qkv[:, heads + kv:], table, lens)
        y = cache.attend(q, table, lens)
        h, r = tsd.residual_norm(x, y.view(n, d), norm="rms", weight=w)
        y = states.attend(h.view(n, heads, dim))
        h, r = tsd.residual_norm(r, y.view(n, d), norm="layer", weight=w, bias=bias, out=(None, r))
        return h, r

    def begin():  # a cache with the tokens before, and its lengths
        cache = tsd.KV8Cache.empty(24, n, kv, dim, block=16, dtype=BF)
        lens = torch.tensor([0, 15, 16], dtype=torch.int32, device="cuda")
        cache.append(rotary.rand(31, kv, dim, seed=5), rotary.rand(31, kv, dim, seed=6), table, lens, starts=cross.ints([0, 0, 15, 31]))
        return cache, lens

    layer(*begin(), x)  # (workspaces' sizes and kernels' attributes are asked for once)
    caches, lens = zip(*(begin() for _ in range(2)))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer(caches[0], lens[0], x)
    for step in range(20):
        qkv.copy_(rotary.rand(n, heads + 2 * kv, dim, seed=100 + step))
        x.copy_(torch.randn(n, d, generator=torch.Generator().manual_seed(step)))
        g.replay()
        want = layer(caches[1], lens[1], x)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), step
    assert torch.equal(lens[0], lens[1])
