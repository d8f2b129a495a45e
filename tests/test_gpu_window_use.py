"""Norm with rotary positions, the cache in pages and attention with a window as a program uses them: captured and
replayed, on other streams, behind 32-bit offsets, beside memory that is not theirs."""
import math

import numpy as np
import pytest

import operators_ref as R
import window_ref as W
from test_gpu_operators import ctx, ints, normal, offsets, spaced  # noqa: F401
from test_gpu_window import new_pages, random_table

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32


# --- one training step and one serving step ---------------------------------------------------------

def train_state(seed, dim=128, lengths=(70, 0, 331, 1), heads=4, kv_heads=2):
    n = sum(lengths)
    s = {name: normal(seed + i, n, h, dim).cuda() for i, (name, h) in enumerate(
        (("xq", heads), ("xk", kv_heads), ("v", kv_heads), ("dout", heads)))}
    for name, like in (("q", "xq"), ("k", "xk"), ("out", "xq"), ("dq", "xq"), ("dk", "xk"), ("dv", "v"), ("dxq", "xq"), ("dxk", "xk")):
        s[name] = torch.full_like(s[like], math.nan)
    s["lse"] = torch.full((heads, n), math.nan, device="cuda")
    s["w"] = [(1 + 0.3 * normal(seed + 7 + i, dim, dtype=F32)).cuda() for i in range(2)]
    s["dw"] = [torch.full((dim,), math.nan, device="cuda") for _ in range(2)]
    s["pos"] = torch.cat([torch.arange(m, dtype=torch.int32) for m in lengths]).view(1, n).cuda()
    s["cu"], s["lengths"], s["dim"] = offsets(lengths), lengths, dim
    return s


OUTS = ("q", "k", "out", "lse", "dq", "dk", "dv", "dxq", "dxk")
MASK = dict(causal_block=1, window=100, sinks=3)


def train_step(ctx, s, **work):
    at = dict(axis_dims=(s["dim"],), positions=s["pos"])
    ctx.norm_rotate((s["xq"], s["xk"]), s["w"], (s["q"], s["k"]), **at)
    ctx.window_attention(s["q"], s["k"], s["v"], s["cu"], out=s["out"], lse=s["lse"], **MASK, **work)
    ctx.window_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["cu"], None, s["dq"], s["dk"], s["dv"],
                                  **MASK, **work)
    ctx.norm_rotate_backward((s["xq"], s["xk"]), s["w"], (s["dq"], s["dk"]), (s["dxq"], s["dxk"]), s["dw"], **at, **work)


def results(s):
    return [s[x].clone() for x in OUTS] + [x.clone() for x in s["dw"]]


def train_reference(s):
    """Every operator against its plain form, on the inputs that it had."""
    pos = s["pos"].cpu()
    for x, w, y, dy, dx, dw in (("xq", 0, "q", "dq", "dxq", 0), ("xk", 1, "k", "dk", "dxk", 1)):
        W.assert_close(s[y], *W.norm_rotate(s[x].cpu(), s["w"][w].cpu(), pos, (s["dim"],), BF), y)
        a, ta, b, tb = W.norm_rotate_backward(s[x].cpu(), s["w"][w].cpu(), s[dy].cpu(), pos, (s["dim"],))
        W.assert_close(s[dx], a, ta, dx)
        W.assert_close(s["dw"][dw], b, tb, "dw")
    at = 0
    for n in s["lengths"]:
        rows = slice(at, at + n)
        q, k, v, do = (s[x][rows].cpu() for x in ("q", "k", "v", "dout"))
        seen = W.sees(n, n, 1, MASK["window"], MASK["sinks"])
        out, mag, _, _ = W.attention(q, k, v, seen)
        W.assert_attention(s["out"][rows], out, mag, "out")
        for name, (g, tol) in W.gradients(q, k, v, do, seen).items():
            W.assert_close(s[name][rows], g, tol, name)
        at += n


@pytest.mark.parametrize("dim", [64, 128])
def test_train_step(ctx, dim):
    s = train_state(500, dim)
    train_step(ctx, s)
    train_reference(s)
    first = results(s)
    train_step(ctx, s)
    for a, b in zip(first, results(s)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dim", [64, 128])
def test_train_step_captured_and_replayed(ctx, dim):
    s, other = train_state(510, dim), train_state(520, dim, (900, 5))
    train_step(ctx, s)
    want = results(s)
    train_step(ctx, other)
    want_other = results(other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train_step(ctx, s)
    for i in range(5):
        for x in OUTS:
            s[x].fill_(math.nan)
            other[x].fill_(math.nan)
        graph.replay()
        train_step(ctx, other)                   # the program's own work between replays
        torch.cuda.synchronize()
        for name, got, w in zip(OUTS + ("dw", "dw"), results(s) + results(other), want + want_other):
            assert torch.equal(got, w), f"replay {i}: {name}"
    # offsets and positions are read at replay
    s["lengths"] = (0, 200, 130, 72)
    s["cu"].copy_(offsets(s["lengths"]))
    s["pos"].copy_(torch.cat([torch.arange(m, dtype=torch.int32) for m in s["lengths"]]).view(1, -1))
    graph.replay()
    torch.cuda.synchronize()
    train_reference(s)


def serve_state(ctx, seed, lengths, kv_heads=2, group=4, dim=128, page=16, per=40):
    s = {"pages": new_pages(ctx, len(lengths) * per, page, kv_heads, dim), "lengths": list(lengths)}
    s["table"] = random_table(seed, len(lengths), per, len(lengths) * per).cuda()
    s["old"] = [[normal(seed + 10 * i + j, m, kv_heads, dim) for j in range(2)] for i, m in enumerate(lengths)]
    cu = offsets(lengths)
    k, v = (torch.cat([o[j] for o in s["old"]]).cuda() for j in range(2))
    ctx.paged_append(s["pages"], s["table"], k, v, ints([0] * len(lengths)), cu)
    n = len(lengths)
    s["q"], s["k"], s["v"] = (normal(seed + 100 + i, n, h, dim).cuda() for i, h in enumerate((kv_heads * group, kv_heads, kv_heads)))
    s["out"] = torch.full_like(s["q"], math.nan)
    s["start"], s["kv_len"] = ints(lengths), ints([m + 1 for m in lengths])
    return s


def serve_step(ctx, s, **work):
    """One new token of every sequence."""
    ctx.paged_append(s["pages"], s["table"], s["k"], s["v"], s["start"])
    ctx.paged_attention(s["pages"], s["table"], s["q"], s["kv_len"], out=s["out"], **MASK, **work)


def serve_reference(s, got=None):
    for b, (m, old) in enumerate(zip(s["lengths"], s["old"])):
        k, v = (torch.cat([o[:m], s[x][b:b + 1].cpu()]) for o, x in zip(old, ("k", "v")))
        out, mag, _, _ = W.attention(s["q"][b:b + 1].cpu(), k, v, W.sees(1, m + 1, 1, MASK["window"], MASK["sinks"]))
        W.assert_attention((s["out"] if got is None else got)[b:b + 1], out, mag, f"sequence {b}")


def test_serving_captured_and_replayed(ctx):
    s, other = serve_state(ctx, 530, [0, 15, 16, 400, 99]), serve_state(ctx, 540, [600] * 3)
    serve_step(ctx, s)
    want = s["out"].clone()
    serve_reference(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve_step(ctx, s)
    for i in range(5):
        s["out"].fill_(math.nan)
        graph.replay()
        serve_step(ctx, other)
        torch.cuda.synchronize()
        assert torch.equal(s["out"], want), f"replay {i}"
    # lengths, slots and tables are read at replay: a token further, in other pages
    for b, old in enumerate(s["old"]):
        s["old"][b] = [torch.cat([o, s[x][b:b + 1].cpu()]) for o, x in zip(old, ("k", "v"))]
    s["lengths"] = [m + 1 for m in s["lengths"]]
    s["start"] += 1
    s["kv_len"] += 1
    moved = s["table"].flip(1).contiguous()                # every sequence's pages in the opposite order
    for t in (s["pages"].k, s["pages"].v):
        t[moved.long()] = t[s["table"].long()].clone()
    s["table"].copy_(moved)
    graph.replay()
    torch.cuda.synchronize()
    serve_reference(s)


def test_graphs_with_workspaces_of_their_own(ctx):
    """Captured calls that need room for partial results, replayed at the same time on two streams."""
    sides = []
    for i in range(2):
        s = train_state(550 + i, 64, (1500,))
        p = serve_state(ctx, 560 + i, [5000], per=320)
        work = [torch.full((32 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]      # NaN

        def call(s=s, p=p, work=work):
            train_step(ctx, s, workspace=work[0])
            ctx.paged_append(p["pages"], p["table"], p["k"], p["v"], p["start"])
            ctx.paged_attention(p["pages"], p["table"], p["q"], p["kv_len"], out=p["out"], workspace=work[1])
        call()
        torch.cuda.synchronize()
        want = results(s) + [p["out"].clone()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        sides.append((graph, s, p, want, torch.cuda.Stream(), call))
    for _ in range(4):
        for _, s, p, *_ in sides:
            for x in OUTS:
                s[x].fill_(math.nan)
            p["out"].fill_(math.nan)
        torch.cuda.synchronize()
        for graph, *_, stream, _ in sides:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, s, p, want, *_ in sides:
            for got, w in zip(results(s) + [p["out"]], want):
                assert torch.equal(got, w)


def test_on_another_stream(ctx):
    s, p = train_state(570), serve_state(ctx, 580, [40, 300])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        train_step(ctx, s)
        serve_step(ctx, p)
    side.synchronize()
    train_reference(s)
    serve_reference(p)


def test_profile_counts(hc):
    c = hc.Context(hc.make_config(n_layers=1), 0)
    s, p = train_state(590), serve_state(c, 600, [40, 300])
    c.profile_enable()
    train_step(c, s)
    serve_step(c, p)
    assert [c.profile_read(k)[1] for k in (hc.K_ROTATE, hc.K_CACHE, hc.K_SEQUENCE, hc.K_GRADIENT)] == [2, 1, 2, 1]
    c.close()


# --- what is not theirs ------------------------------------------------------------------------------

@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lengths", [(33, 64, 100), (1000, 1100)])
def test_rows_outside_are_left_and_not_seen(ctx, dim, lengths):
    """Rows before the first and behind the last sequence hold NaN and stay as they were; another sequence's NaN stays
    its own."""
    heads, kv_heads, before, behind = 2, 1, 3, 70
    total = before + sum(lengths) + behind
    cu = ints([before] + (before + np.cumsum(lengths)).tolist())
    q, k, v, do = (torch.full((total, h, dim), math.nan, dtype=BF, device="cuda") for h in (heads, kv_heads, kv_heads, heads))
    own = slice(before, total - behind)
    host = [normal(610 + i, sum(lengths), t.shape[1], dim) for i, t in enumerate((q, k, v, do))]
    for t, h in zip((q, k, v, do), host):
        t[own] = h.cuda()
    sick = before + lengths[0]                             # the second sequence, all of it
    for t in (q, k, v, do):
        t[sick:sick + lengths[1]] = math.nan
    out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, q, k, v))
    lse = torch.full((heads, total), 7.0, device="cuda")
    kw = dict(causal_block=1, window=50, sinks=2)
    ctx.window_attention(q, k, v, cu, out=out, lse=lse, **kw)
    ctx.window_attention_backward(q, k, v, out, lse, do, cu, None, dq, dk, dv, **kw)
    for t in (out, dq, dk, dv, lse.t()):
        assert bool((t[:before] == 7.0).all()) and bool((t[total - behind:] == 7.0).all())
    at = 0
    for i, n in enumerate(lengths):
        rows, mine = slice(at, at + n), slice(before + at, before + at + n)
        at += n
        if i == 1:
            continue
        hq, hk, hv, hdo = (t[rows] for t in host)
        seen = W.sees(n, n, 1, 50, 2)
        want, mag, _, _ = W.attention(hq, hk, hv, seen)
        W.assert_attention(out[mine], want, mag, "out")
        for t, (g, tol) in zip((dq, dk, dv), W.gradients(hq, hk, hv, hdo, seen).values()):
            W.assert_close(t[mine], g, tol, "gradient")


@pytest.mark.parametrize("dim,queries", [(128, 1), (64, 3), (64, 120), (128, 600)])
def test_pages_of_others_and_rows_outside(ctx, dim, queries):
    """A sequence whose pages hold NaN beside one that is well; query rows that belong to no sequence."""
    m, heads = 700, 2
    pages = new_pages(ctx, 100, 16, heads, dim)
    table = random_table(11, 2, 44, 100).cuda()
    k, v, q = normal(620, m, heads, dim), normal(621, m, heads, dim), normal(622, queries, heads, dim)
    ctx.paged_append(pages, table[:1].contiguous(), k.cuda(), v.cuda(), ints([0]))
    qs = torch.full((2 * queries + 5, heads, dim), math.nan, dtype=BF, device="cuda")
    qs[:queries] = q.cuda()
    out = torch.full_like(qs, 7.0)
    ctx.paged_attention(pages, table, qs, ints([m, m]), ints([0, queries, 2 * queries]), out, window=90)
    want, mag, _, _ = W.attention(q, k, v, W.sees(queries, m, 1, 90, 0))
    W.assert_attention(out[:queries], want, mag, "the well one")
    assert bool((out[2 * queries:] == 7.0).all()) and not bool((out[queries:2 * queries] == 7.0).any())


def test_lengths_outside_the_slots(ctx):
    """kv_len is clamped to the table's slots, below and above."""
    k, v, q = normal(623, 48, 2, 64), normal(624, 48, 2, 64), normal(625, 3, 2, 64)
    pages, table = new_pages(ctx, 9, 16, 2, 64), random_table(12, 3, 3, 9).cuda()
    ctx.paged_append(pages, table, torch.cat([k] * 3).cuda(), torch.cat([v] * 3).cuda(), ints([0, 0, 0]), ints([0, 48, 96, 144]))
    got = ctx.paged_attention(pages, table, q.cuda(), ints([2147483647, -5, 48]))
    for i in (0, 2):
        want, mag, _, _ = W.attention(q[i:i + 1], k, v, W.sees(1, 48, 1, 0, 0))
        W.assert_attention(got[i:i + 1], want, mag, f"sequence {i}")
    assert not bool(got[1].any())


# --- sizes ------------------------------------------------------------------------------------------

def test_nothing_to_do(ctx):
    none, keys = torch.zeros(0, 2, 64, dtype=BF, device="cuda"), normal(630, 5, 2, 64).cuda()
    kw = dict(axis_dims=(64,), positions=torch.zeros(1, 0, dtype=torch.int32, device="cuda"))
    w = torch.ones(64, device="cuda")
    assert ctx.norm_rotate(none, w, **kw).shape == none.shape
    dx, dw = ctx.norm_rotate_backward(none, w, none, None, torch.full((64,), math.nan, device="cuda"), **kw)
    assert not bool(dw.any())
    pages = new_pages(ctx, 2, 16, 2, 64, fill=7.0)
    table = ints([[0, 1]])
    ctx.paged_append(pages, table, none, none, ints([0]))
    assert bool((pages.k == 7.0).all()) and ctx.paged_attention(pages, table, none, ints([0])).shape == none.shape
    # keys without queries get zeros, queries without keys too
    lse = torch.zeros(2, 0, device="cuda")
    cu = ints([0, 0]), ints([0, 5])
    out = ctx.window_attention(none, keys, keys.clone(), *cu, lse=lse)
    dq, dk, dv = ctx.window_attention_backward(none, keys, keys.clone(), out, lse, none, *cu)
    assert dq.shape == none.shape and not bool(dk.any()) and not bool(dv.any())
    lse = torch.zeros(2, 5, device="cuda")
    cu = cu[::-1]
    out = ctx.window_attention(keys, none, none.clone(), *cu, lse=lse)
    dq, dk, dv = ctx.window_attention_backward(keys, none, none.clone(), out, lse, keys.clone(), *cu)
    assert not bool(out.any()) and not bool(dq.any()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dim", [64, 128])
def test_thousands_of_short_sequences(ctx, dim):
    """More sequences than a work group's threads: every one is found, empty ones between them."""
    lengths = (np.arange(3000) % 5).tolist()
    n, heads = sum(lengths), 2
    q, k, v, do = (normal(640 + i, n, heads, dim) for i in range(4))
    cu = offsets(lengths)
    d = [t.cuda() for t in (q, k, v, do)]
    lse = torch.empty(heads, n, device="cuda")
    out = ctx.window_attention(*d[:3], cu, lse=lse, window=3)
    grads = ctx.window_attention_backward(*d[:3], out, lse, d[3], cu, window=3)
    # sequences of one length at once, as heads of one
    for m in range(1, 5):
        rows = torch.tensor([i for s, at in enumerate(np.cumsum([0] + lengths)[:-1]) if lengths[s] == m for i in range(at, at + m)])
        fold = lambda t: t[rows].view(-1, m, heads, dim).transpose(0, 1).reshape(m, -1, dim)  # noqa: E731, B023
        qs, ks, vs, dos = (fold(t) for t in (q, k, v, do))
        seen = W.sees(m, m, 1, 3, 0)
        want, mag, _, _ = W.attention(qs, ks, vs, seen)
        W.assert_attention(fold(out.cpu()), want, mag, f"length {m}")
        for t, (name, (g, tol)) in zip(grads, W.gradients(qs, ks, vs, dos, seen).items()):
            W.assert_close(fold(t.cpu()), g, tol, f"{name}, length {m}")
    # and the same through pages, a page each
    pages, table = new_pages(ctx, 3000, 16, heads, dim), torch.arange(3000, dtype=torch.int32, device="cuda").view(3000, 1)
    ctx.paged_append(pages, table, d[1], d[2], torch.zeros(3000, dtype=torch.int32, device="cuda"), cu)
    got = ctx.paged_attention(pages, table, d[0], ints(lengths), cu, window=3)
    assert bool(((got - out).abs() <= 2.0 ** -6 * d[2].abs().max()).all())


def test_shared_rows(ctx):
    """Inputs broadcast along tokens or heads: gradients are of every row by itself."""
    n, heads, dim = 200, 3, 64
    q, k, v, do = normal(650, n, 1, dim), normal(651, n, 1, dim), normal(652, 1, 1, dim), normal(653, 1, heads, dim)
    args = [t.cuda().expand(n, h, dim) for t, h in ((q, heads), (k, heads), (v, heads), (do, heads))]
    lse = torch.empty(heads, n, device="cuda")
    out = ctx.window_attention(*args[:3], lse=lse, window=40, sinks=1)
    grads = ctx.window_attention_backward(*args[:3], out, lse, args[3], window=40, sinks=1)
    host = [t.cpu() for t in args]
    seen = W.sees(n, n, 1, 40, 1)
    W.assert_attention(out, *W.attention(*host[:3], seen)[:2], "out")
    for t, (name, (g, tol)) in zip(grads, W.gradients(*host, seen).items()):
        W.assert_close(t, g, tol, name)
    pos = torch.arange(n, dtype=torch.int32).view(1, n)
    w = normal(654, dim, dtype=F32)
    y = ctx.norm_rotate(args[0], w.cuda(), axis_dims=(dim,), positions=pos.cuda())
    W.assert_close(y, *W.norm_rotate(host[0], w, pos, (dim,), BF), "y")
    dx, dw = ctx.norm_rotate_backward(args[0], w.cuda(), args[3], axis_dims=(dim,), positions=pos.cuda())
    a, ta, b, tb = W.norm_rotate_backward(host[0], w, host[3], pos, (dim,))
    W.assert_close(dx, a, ta, "dx")
    W.assert_close(dw, b, tb, "dw")


def test_one_head_of_many_tokens_and_many_heads_of_one(ctx):
    for n, heads in ((20000, 1), (1, 5000)):
        x = normal(655, n, heads, 64)
        w = 1 + 0.3 * normal(656, 64, dtype=F32)
        pos = torch.arange(n, dtype=torch.int32).view(1, n) * 7
        kw = dict(axis_dims=(64,), positions=pos.cuda())
        W.assert_close(ctx.norm_rotate(x.cuda(), w.cuda(), **kw), *W.norm_rotate(x, w, pos, (64,), BF), "y")
        g = normal(657, n, heads, 64)
        dx, dw = ctx.norm_rotate_backward(x.cuda(), w.cuda(), g.cuda(), **kw)
        a, ta, b, tb = W.norm_rotate_backward(x, w, g, pos, (64,))
        W.assert_close(dx, a, ta, "dx")
        W.assert_close(dw, b, tb, "dw")


# --- offsets that pass 32 bits ------------------------------------------------------------------------

@pytest.mark.parametrize("dim", [64, 128])
def test_pages_behind_32_bit_offsets(ctx, dim):
    n_pages, page, heads = (1 << 32) // (64 * 4 * dim) + 40, 64, 4
    pages = new_pages(ctx, n_pages, page, heads, dim, fill=0.0)
    assert pages.k.numel() > 1 << 32
    m = 500
    k, v = normal(660, m, heads, dim), normal(661, m, heads, dim)
    table = torch.arange(n_pages - 8, n_pages, dtype=torch.int32, device="cuda").view(1, 8)
    ctx.paged_append(pages, table, k.cuda(), v.cuda(), ints([0]))
    assert torch.equal(pages.k[n_pages - 1, :m - 448].cpu(), k[448:])
    for queries in (1, 90, 400):
        q = normal(662, queries, heads * 2, dim)
        got = ctx.paged_attention(pages, table, q.cuda(), ints([m]), window=300, sinks=20)
        want, mag, _, _ = W.attention(q, k, v, W.sees(queries, m, 1, 300, 20))
        W.assert_attention(got, want, mag, f"{queries} queries")


@pytest.mark.parametrize("dim", [64, 128])
def test_rows_behind_32_bit_offsets(ctx, dim):
    """Tokens 2^23 elements apart: 600 of them pass 2^32 elements."""
    n, far = 600, 1 << 23
    big = torch.empty(n * far, dtype=BF, device="cuda")
    place = iter(range(0, 1 << 20, 1 << 10))

    def put(t):
        view = big.as_strided(t.shape, (far, dim, 1), next(place))
        view.copy_(t)
        return view
    q, k, v, do = (normal(670 + i, n, h, dim) for i, h in enumerate((4, 2, 2, 4)))
    d = [put(t) for t in (q, k, v, do)]
    out, dq, dk, dv, y, dx = (put(torch.zeros_like(t)) for t in (q, q, k, v, q, q))
    lse = torch.empty(4, n, device="cuda")
    kw = dict(window=200, sinks=9)
    ctx.window_attention(*d[:3], out=out, lse=lse, **kw)
    ctx.window_attention_backward(*d[:3], out, lse, d[3], None, None, dq, dk, dv, **kw)
    seen = W.sees(n, n, 1, 200, 9)
    want, mag, _, _ = W.attention(q, k, v, seen)
    W.assert_attention(out, want, mag, "out")
    for t, (name, (g, tol)) in zip((dq, dk, dv), W.gradients(q, k, v, do, seen).items()):
        W.assert_close(t, g, tol, name)
    pos, w = torch.arange(n, dtype=torch.int32).view(1, n), 1 + 0.3 * normal(675, dim, dtype=F32)
    at = dict(axis_dims=(dim,), positions=pos.cuda())
    ctx.norm_rotate(d[0], w.cuda(), y, **at)
    W.assert_close(y, *W.norm_rotate(q, w, pos, (dim,), BF), "y")
    _, dw = ctx.norm_rotate_backward(d[0], w.cuda(), d[3], dx, **at)
    a, ta, b, tb = W.norm_rotate_backward(q, w, do, pos, (dim,))
    W.assert_close(dx, a, ta, "dx")
    W.assert_close(dw, b, tb, "dw")


@pytest.mark.parametrize("dim", [64, 128])
def test_a_key_head_of_many(ctx, dim):
    """More query heads on a key head than a unit has rows."""
    for group, queries, keys in ((150, [3, 20], [40, 20]), (300, [1], [70])):
        q, k, v, do = (normal(680 + i, sum(n), h, dim) for i, (n, h) in enumerate(((queries, group), (keys, 1), (keys, 1), (queries, group))))
        d = [t.cuda() for t in (q, k, v, do)]
        cu = offsets(queries), offsets(keys)
        lse = torch.empty(group, sum(queries), device="cuda")
        out = ctx.window_attention(*d[:3], *cu, lse=lse, window=17, sinks=2)
        grads = ctx.window_attention_backward(*d[:3], out, lse, d[3], *cu, window=17, sinks=2)
        pages, table = new_pages(ctx, 20, 16, 1, dim), random_table(13, len(keys), 5, 20).cuda()
        ctx.paged_append(pages, table, d[1], d[2], ints([0] * len(keys)), cu[1])
        paged = ctx.paged_attention(pages, table, d[0], ints(keys), cu[0], window=17, sinks=2)
        a = b = 0
        for n, m in zip(queries, keys):
            qs, ks, vs, dos = q[a:a + n], k[b:b + m], v[b:b + m], do[a:a + n]
            seen = W.sees(n, m, 1, 17, 2)
            want, mag, _, _ = W.attention(qs, ks, vs, seen)
            W.assert_attention(out[a:a + n], want, mag, "out")
            W.assert_attention(paged[a:a + n], want, mag, "pages")
            for t, (name, (g, tol)) in zip(grads, W.gradients(qs, ks, vs, dos, seen).items()):
                lo, hi = (a, a + n) if name == "dq" else (b, b + m)
                W.assert_close(t[lo:hi], g, tol, name)
            a, b = a + n, b + m


@pytest.mark.parametrize("dim", [64, 128])
def test_scales(ctx, dim):
    """A scale of the caller's, small and large."""
    n = 150
    q, k, v, do = (normal(690 + i, n, 2, dim) for i in range(4))
    d = [t.cuda() for t in (q, k, v, do)]
    seen = W.sees(n, n, 1, 60, 1)
    for scale in (1e-20, 0.01, 0.6):
        lse = torch.empty(2, n, device="cuda")
        kw = dict(window=60, sinks=1, softmax_scale=scale)
        out = ctx.window_attention(*d[:3], lse=lse, **kw)
        W.assert_attention(out, *W.attention(q, k, v, seen, scale)[:2], f"scale {scale}")
        grads = ctx.window_attention_backward(*d[:3], out, lse, d[3], **kw)
        for t, (name, (g, tol)) in zip(grads, W.gradients(q, k, v, do, seen, scale).items()):
            W.assert_close(t, g, tol, f"{name}, scale {scale}")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("queries,keys", [(1, 700), (40, 3000), (300, 1500), (5, 20000)])
def test_logarithms_of_merged_ranges(ctx, dim, queries, keys):
    """Few rows over many keys are cut into ranges: the logarithms of the whole rows, and gradients from them."""
    q, k, v, do = (normal(700 + i, n, h, dim) for i, (n, h) in enumerate(((queries, 4), (keys, 2), (keys, 2), (queries, 4))))
    d = [t.cuda() for t in (q, k, v, do)]
    cu = offsets([queries]), offsets([keys])
    for window, sinks in ((0, 0), (keys // 2, 100)):
        seen = W.sees(queries, keys, 1, window, sinks)
        lse = torch.full((4, queries), math.nan, device="cuda")
        kw = dict(window=window, sinks=sinks)
        out = ctx.window_attention(*d[:3], *cu, lse=lse, **kw)
        want, mag, logs, _ = W.attention(q, k, v, seen)
        W.assert_attention(out, want, mag, "out")
        assert bool(((lse.cpu().double() - logs).abs() <= 2.0 ** -8 * 1.02).all())
        grads = ctx.window_attention_backward(*d[:3], out, lse, d[3], *cu, **kw)
        for t, (name, (g, tol)) in zip(grads, W.gradients(q, k, v, do, seen).items()):
            W.assert_close(t, g, tol, name)


@pytest.mark.parametrize("dim", [64, 128])
def test_gradients_of_large_logits(ctx, dim):
    """Logits of several hundreds: rows that a few keys carry, and whose logarithms are large.

    Forming p again, a logit is off by 2^-24 of the sum of its products' magnitudes for each of the up to 8 products
    along its dims, the logarithm by as much once more: 2^-20 of that sum in all, which scales every tolerance's 2^-7."""
    n = 420
    q, k = (normal(720 + i, n, 2, dim, spread=8.0) for i in range(2))
    v, do = (normal(722 + i, n, 2, dim) for i in range(2))
    d = [t.cuda() for t in (q, k, v, do)]
    for window, sinks in ((0, 0), (90, 6)):
        seen = W.sees(n, n, 1, window, sinks)
        size = float((q.double().abs().transpose(0, 1) @ k.double().abs().permute(1, 2, 0)).max()) * dim ** -0.5
        lse = torch.empty(2, n, device="cuda")
        out = ctx.window_attention(*d[:3], lse=lse, window=window, sinks=sinks)
        grads = ctx.window_attention_backward(*d[:3], out, lse, d[3], window=window, sinks=sinks)
        for t, (name, (g, tol)) in zip(grads, W.gradients(q, k, v, do, seen).items()):
            W.assert_close(t, g, tol * (1 + size * 2.0 ** -20 / 2.0 ** -7), name)
