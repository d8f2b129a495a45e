"""Norm with rotary positions, the cache in pages with its attention, and attention with a window and its
gradients, on the GPU against the plain 64-bit forms of tests/window_ref.py."""
import math

import numpy as np
import pytest

import operators_ref as R
import window_ref as W
from test_gpu_operators import ctx, ints, normal, offsets, spaced  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32


# --- norm and rotary positions ---------------------------------------------------------------------

NORM = [
    # tokens, heads, dim, axis_dims, halves, joint, inverse, input, output, weight, far
    (1, 1, 64, (64,), False, False, False, BF, BF, BF, 1 << 20),
    (1, 12, 128, (44, 42, 42), False, False, False, BF, BF, F32, 0),
    (130, 3, 128, (44, 42, 42), False, False, True, BF, F32, BF, 0),
    (77, 5, 64, (24, 20, 20), True, True, False, BF, BF, BF, 0),
    (500, 2, 128, (16, 56, 56), True, False, False, F32, F32, F32, 2147483647),
    (33, 4, 96, (16, 16, 16), False, True, True, F32, F32, None, 1 << 20),      # dims behind the rotated ones
    (33, 4, 96, (16, 16, 16), True, False, False, F32, BF, F32, 1000),
    (9, 7, 256, (64, 64, 64, 64), True, True, False, F32, F32, BF, 5000),
    (9, 7, 256, (250, 0, 4, 2), False, False, True, F32, F32, F32, 5000),
    (5, 1, 16, (6, 4, 6), True, False, False, F32, F32, F32, 99),
    (7, 9, 248, (16,), True, False, False, BF, BF, BF, 99),                      # 30 of 32 lanes
    (12, 3, 24, (16,), False, False, True, BF, F32, None, 7),                    # 3 of 4 lanes
    (1030, 3, 128, (64, 64), False, False, False, BF, BF, BF, 1 << 30),
]
NORM_IDS = [f"{c[0]}x{c[1]}x{c[2]}_{len(c[3])}ax{'_halves' if c[4] else ''}" for c in NORM]


def norm_case(case, seed):
    n, heads, d, axes, halves, joint, inverse, xt, ot, wt, far = case
    spread = torch.exp(normal(seed, 1, heads, 1, dtype=F32))
    x = (normal(seed + 1, n, heads, d, dtype=F32) * spread).to(xt)
    w = None if wt is None else (1 + 0.3 * normal(seed + 2, d, dtype=F32)).to(wt)
    if far:
        pos = torch.from_numpy(np.random.default_rng(3).integers(-far, far, (len(axes), n), dtype=np.int64))
        at = dict(positions=pos.to(torch.int32).cuda())
    else:
        pos = R.grid_positions(n, 7, 9, 41)
        at = dict(grid=(7, 9), frame0=41)
    kw = dict(halves=halves, joint=joint, inverse=inverse)
    return x, w, pos, dict(axis_dims=axes, **kw, **at), kw


@pytest.mark.parametrize("case", NORM, ids=NORM_IDS)
def test_norm_rotate(ctx, case):
    n, heads, d, axes, *_, ot, wt, far = case
    x, w, pos, call, kw = norm_case(case, 20)
    want, tol = W.norm_rotate(x, w, pos, axes, ot, **kw)
    out = torch.full((heads, n, d), math.nan, dtype=ot, device="cuda").transpose(0, 1)      # head-major
    ctx.norm_rotate(spaced(x), None if w is None else w.cuda(), out, **call)
    W.assert_close(out, want, tol, "y")


@pytest.mark.parametrize("case", NORM, ids=NORM_IDS)
def test_norm_rotate_backward(ctx, case):
    n, heads, d, axes, *_, ot, wt, far = case
    x, w, pos, call, kw = norm_case(case, 30)
    dout = normal(33, n, heads, d, dtype=ot)
    dx, tol, dw, tol_w = W.norm_rotate_backward(x, w, dout, pos, axes, **kw)
    got = torch.full((heads, n, d), math.nan, dtype=x.dtype, device="cuda").transpose(0, 1)
    gw = torch.full((d,), math.nan, dtype=F32, device="cuda")
    ctx.norm_rotate_backward(spaced(x), None if w is None else w.cuda(), spaced(dout), got, gw, **call)
    W.assert_close(got, dx, tol, "dx")
    W.assert_close(gw, dw, tol_w, "dw")


@pytest.mark.parametrize("n", [1, 63, 1500])
@pytest.mark.parametrize("halves", [False, True])
def test_norm_pair_in_place(ctx, n, halves):
    q, k = normal(4, n, 12, 128), normal(5, n, 3, 128)
    ws = [(1 + 0.3 * normal(6 + i, 128, dtype=F32)).to(BF) for i in range(2)]
    dws = [w.cuda() for w in ws]
    pos = R.grid_positions(n, 30, 52, 0)
    dq, dk = q.cuda(), spaced(k)
    got = ctx.norm_rotate((dq, dk), dws, (dq, dk), axis_dims=(44, 42, 42), halves=halves)       # the context's grid
    assert got[0] is dq and got[1] is dk
    for name, t, x, w in (("q", dq, q, ws[0]), ("k", dk, k, ws[1])):
        W.assert_close(t, *W.norm_rotate(x, w, pos, (44, 42, 42), BF, halves=halves), name)
    gq, gk = normal(8, n, 12, 128), normal(9, n, 3, 128)
    rq, rk = gq.cuda(), gk.cuda()
    (xq, xk), (wq, wk) = ctx.norm_rotate_backward((q.cuda(), k.cuda()), dws, (rq, rk), (rq, rk), axis_dims=(44, 42, 42), halves=halves)
    assert xq is rq and xk is rk                       # in the place of the output's gradients
    for name, x, w, g, dx, dw in (("q", q, ws[0], gq, xq, wq), ("k", k, ws[1], gk, xk, wk)):
        a, ta, b, tb = W.norm_rotate_backward(x, w, g, pos, (44, 42, 42), halves=halves)
        W.assert_close(dx, a, ta, "d" + name)
        W.assert_close(dw, b, tb, "dw" + name)


def test_norm_gradient_is_the_difference(ctx):
    """Central differences of the library's own forward pass, in 32 bits."""
    n, heads, d, axes = 6, 2, 64, (24, 20, 20)
    x, w, g = (normal(s, *shape, dtype=F32).cuda() for s, shape in ((40, (n, heads, d)), (41, (d,)), (42, (n, heads, d))))
    kw = dict(axis_dims=axes, grid=(2, 2), frame0=3)
    dx, dw = ctx.norm_rotate_backward(x, w, g, **kw)
    y = lambda x, w: (ctx.norm_rotate(x, w, **kw).double() * g.double()).sum()  # noqa: E731
    step = 2.0 ** -6
    along_x, along_w = normal(43, n, heads, d, dtype=F32).cuda(), normal(44, d, dtype=F32).cuda()
    by_x = (y(x + step * along_x, w) - y(x - step * along_x, w)) / (2 * step)
    by_w = (y(x, w + step * along_w) - y(x, w - step * along_w)) / (2 * step)
    # the third derivative's term: step^2 of the value; 32-bit outputs: 2^-21 of the sums' size over the step
    size = float(g.abs().double().sum()) * 4
    assert abs(float(by_x - (dx.double() * along_x.double()).sum())) <= size * (step ** 2 + 2.0 ** -21 / step)
    assert abs(float(by_w - (dw.double() * along_w.double()).sum())) <= size * (step ** 2 + 2.0 ** -21 / step)


def test_norm_of_zeros_and_large_values(ctx):
    x = torch.zeros(4, 2, 64, dtype=F32)
    x[1] = 1e18                                        # the sum of squares is still in range
    x[2, 0, 3] = math.nan
    x[3, 1, 5] = 1e-30
    w = torch.ones(64, device="cuda")
    got = ctx.norm_rotate(x.cuda(), w, axis_dims=(64,), positions=ints([[0, 0, 0, 0]])).cpu()
    assert bool((got[0] == 0).all())
    assert torch.allclose(got[1], torch.ones(2, 64), rtol=1e-6)
    assert torch.isnan(got[2, 0]).all() and bool((got[2, 1] == 0).all())
    assert torch.isfinite(got[3]).all()


# --- pages --------------------------------------------------------------------------------------

def new_pages(ctx, n_pages, page, heads, dim, head_major=True, fill=math.nan):
    if head_major:
        pages = ctx.pages(n_pages, page, heads, dim)
    else:
        k, v = (torch.empty(n_pages, page, heads + 1, dim, dtype=BF, device="cuda")[:, :, :heads] for _ in range(2))
        from paper_2607_20125_amd import headcast
        pages = headcast.Pages(k, v)
    pages.k.fill_(fill)
    pages.v.fill_(fill)
    return pages


def random_table(seed, seqs, per, n_pages):
    return torch.from_numpy(np.random.default_rng(seed).permutation(n_pages)[:seqs * per].astype(np.int32)).view(seqs, per)


@pytest.mark.parametrize("lengths,heads,dim,page,per,head_major,by_offsets", [
    ([1], 1, 128, 16, 1, True, False), ([65], 3, 64, 32, 5, False, True), ([0, 17, 130], 3, 128, 64, 4, True, True),
    ([1] * 64, 8, 64, 16, 3, True, False), ([3] * 70, 2, 128, 16, 9, False, True), ([300, 0, 0, 41], 5, 64, 256, 2, True, True),
    ([2] * 300, 1, 64, 16, 2, True, True)])
def test_paged_append(ctx, lengths, heads, dim, page, per, head_major, by_offsets):
    seqs, total = len(lengths), sum(lengths)
    k, v = normal(50, total, heads, dim), normal(51, total, heads, dim)
    n_pages = seqs * per + 2
    table = random_table(52, seqs, per, n_pages)
    table[0, per - 1] = -1 if seqs > 1 else table[0, per - 1]              # a page that is absent
    start = torch.from_numpy(np.random.default_rng(53).integers(-3, page * per - 1, seqs).astype(np.int32))
    pages = new_pages(ctx, n_pages, page, heads, dim, head_major, 7.0)
    want_k, want_v = pages.k.cpu(), pages.v.cpu()
    at = 0
    for s, n in enumerate(lengths):
        for i in range(n):
            slot = int(start[s]) + i
            if 0 <= slot < page * per and int(table[s, slot // page]) >= 0:
                want_k[table[s, slot // page], slot % page] = k[at + i]
                want_v[table[s, slot // page], slot % page] = v[at + i]
        at += n
    ctx.paged_append(pages, table.cuda(), spaced(k), spaced(v), start.cuda(), offsets(lengths) if by_offsets else None)
    assert torch.equal(pages.k.cpu(), want_k) and torch.equal(pages.v.cpu(), want_v)


def test_paged_append_bad_pages_and_starts(ctx):
    k, v = normal(54, 40, 2, 64), normal(55, 40, 2, 64)
    pages = new_pages(ctx, 3, 16, 2, 64, fill=7.0)
    far = 2147483647
    table = ints([[1, far, -far, 3]])                   # only the first is a page
    for start in (0, 12, 64, -40, far, -far - 1):
        ctx.paged_append(pages, table, k.cuda(), v.cuda(), ints([start]))
    want = torch.full((3, 16, 2, 64), 7.0, dtype=BF)
    want[1] = k[:16]
    want[1, 12:] = k[:4]
    assert torch.equal(pages.k.cpu(), want)


MASKS = [(0, 0, 0), (1, 0, 0), (1, 1, 0), (1, 40, 0), (1, 100, 7), (1, 130, 200), (37, 0, 5), (37, 74, 0), (37, 37, 37), (64, 128, 64)]


def fill_pages(ctx, k, v, lengths, page, seed, gone=()):
    """Pages that hold sequences' keys and values [m][heads][d]; everything else NaN."""
    per = max(1, max(-(-m // page) for m in lengths))
    n_pages = len(lengths) * per + 1
    table = random_table(seed, len(lengths), per, n_pages)
    for s, m in enumerate(lengths):
        table[s, -(-m // page):] = -1                   # nothing behind the end
    for s, p in gone:
        table[s, p] = -1 if p % 2 else n_pages + p
    pages = new_pages(ctx, n_pages, page, k[0].shape[1], k[0].shape[2])
    for s, m in enumerate(lengths):
        for p in range(-(-m // page)):
            at = int(table[s, p])
            if 0 <= at < n_pages:
                rows = slice(p * page, min(m, (p + 1) * page))
                pages.k[at, :rows.stop - rows.start] = k[s][rows].cuda()
                pages.v[at, :rows.stop - rows.start] = v[s][rows].cuda()
    return pages, table.cuda()


@pytest.mark.parametrize("mask", MASKS, ids=lambda m: "block%d_window%d_sinks%d" % m)
@pytest.mark.parametrize("dim,page,group,queries,lengths", [
    (128, 16, 4, [1, 1, 1, 1, 1], [1, 17, 64, 333, 0]),       # single tokens
    (64, 64, 7, [1, 1, 1], [300, 63, 129]),
    (64, 16, 1, [5, 30, 1, 0], [5, 400, 1, 90]),              # few rows, several units
    (128, 32, 2, [70, 200, 3], [70, 517, 2]),                 # chunks, one longer than its keys
    (64, 16, 3, [150, 90], [402, 91]),
])
def test_paged_attention(ctx, mask, dim, page, group, queries, lengths):
    kv_heads = 2
    k, v = ([normal(60 + s + o, m, kv_heads, dim) for s, m in enumerate(lengths)] for o in (0, 20))
    q = [normal(100 + s, n, kv_heads * group, dim) for s, n in enumerate(queries)]
    pages, table = fill_pages(ctx, k, v, lengths, page, 3)
    block, window, sinks = mask
    got = ctx.paged_attention(pages, table, spaced(torch.cat(q)), ints(lengths), offsets(queries), causal_block=block, window=window,
                              sinks=sinks).cpu()
    at = 0
    for s, (n, m) in enumerate(zip(queries, lengths)):
        out, mag, _, _ = W.attention(q[s], k[s], v[s], W.sees(n, m, block, window, sinks))
        W.assert_attention(got[at:at + n], out, mag, f"sequence {s}")
        at += n


@pytest.mark.parametrize("dim,queries,page", [(128, 1, 16), (64, 1, 32), (128, 100, 16), (64, 100, 16), (128, 100, 128)])
def test_paged_attention_absent_pages(ctx, dim, queries, page):
    """Keys of absent pages are hidden, also in the middle of what a query sees, whatever the pages hold."""
    m, heads = 700, 2
    k, v, q = normal(61, m, heads, dim), normal(62, m, heads, dim), normal(63, queries, heads, dim)
    gone = [(0, p) for p in (1, 2, m // page)]
    pages, table = fill_pages(ctx, [k], [v], [m], page, 4, gone)
    mask = W.sees(queries, m, 1, 0, 0)
    for _, p in gone:
        mask[:, p * page:(p + 1) * page] = False
    out, mag, _, _ = W.attention(q, k, v, mask)
    W.assert_attention(ctx.paged_attention(pages, table, q.cuda(), ints([m])), out, mag, "absent")
    table.fill_(-1)
    assert not bool(ctx.paged_attention(pages, table, q.cuda(), ints([m])).any())


def test_paged_long_cache_in_ranges(ctx):
    """One token over a long cache: key ranges, merged; and the same split over many sequences."""
    m, heads, group = 20000, 2, 4
    k, v, q = normal(64, m, heads, 128), normal(65, m, heads, 128), normal(66, 1, heads * group, 128)
    pages, table = fill_pages(ctx, [k], [v], [m], 64, 5)
    for window, sinks in ((0, 0), (9000, 70), (64, 0)):
        out, mag, _, _ = W.attention(q, k, v, W.sees(1, m, 1, window, sinks))
        W.assert_attention(ctx.paged_attention(pages, table, q.cuda(), ints([m]), window=window, sinks=sinks), out, mag, f"window {window}")


def test_paged_large_logits(ctx):
    """Rows whose logits leave the range of a fixed offset, in both kernels."""
    m = 300
    for n in (1, 120):
        k, v, q = normal(67, m, 1, 128, spread=30.0), normal(68, m, 1, 128), normal(69, n, 1, 128, spread=30.0)
        pages, table = fill_pages(ctx, [k], [v], [m], 16, 6)
        got = ctx.paged_attention(pages, table, q.cuda(), ints([m]), window=200, sinks=3)
        out, mag, _, _ = W.attention(q, k, v, W.sees(n, m, 1, 200, 3))
        W.assert_attention(got, out, mag, f"{n} rows")


# --- packed sequences ---------------------------------------------------------------------------

SHAPES = [
    # dim, kv heads, group, queries, keys (None: the queries')
    (64, 1, 1, [1], None),
    (128, 2, 1, [77], None),
    (64, 2, 3, [5, 200, 0, 64, 1], None),
    (128, 1, 4, [130, 40], [300, 7]),            # kept context; fewer keys than queries
    (128, 2, 2, [257, 1, 129], None),
    (64, 1, 2, [100, 3], [0, 250]),              # nothing to see
]


@pytest.mark.parametrize("mask", MASKS, ids=lambda m: "block%d_window%d_sinks%d" % m)
@pytest.mark.parametrize("dim,kv_heads,group,queries,keys", SHAPES, ids=lambda x: str(x).replace(" ", ""))
def test_window_attention_and_gradients(ctx, mask, dim, kv_heads, group, queries, keys):
    block, window, sinks = mask
    lengths = keys or queries
    q, k, v, do = (normal(70 + i, sum(n), h, dim) for i, (n, h) in enumerate(
        ((queries, kv_heads * group), (lengths, kv_heads), (lengths, kv_heads), (queries, kv_heads * group))))
    dq, dk, dv, ddo = (spaced(t) for t in (q, k, v, do))
    cu_q, cu_k = offsets(queries), offsets(lengths) if keys else None
    kw = dict(causal_block=block, window=window, sinks=sinks)
    lse = torch.full((kv_heads * group, sum(queries)), math.nan, device="cuda")
    out = ctx.window_attention(dq, dk, dv, cu_q, cu_k, lse=lse, **kw)
    grads = ctx.window_attention_backward(dq, dk, dv, out, lse, ddo, cu_q, cu_k, **kw)
    again = ctx.window_attention_backward(dq, dk, dv, out, lse, ddo, cu_q, cu_k, **kw)
    a = b = 0
    for s, (n, m) in enumerate(zip(queries, lengths)):
        qs, ks, vs, dos = q[a:a + n], k[b:b + m], v[b:b + m], do[a:a + n]
        seen = W.sees(n, m, block, window, sinks)
        want, mag, logs, _ = W.attention(qs, ks, vs, seen)
        W.assert_attention(out[a:a + n], want, mag, f"sequence {s}")
        got = lse[:, a:a + n].cpu().double()
        assert torch.equal(torch.isinf(got), torch.isinf(logs)) and bool((torch.nan_to_num(got - logs, nan=0.0).abs() <= 2.0 ** -8 * 1.02).all())
        for i, (name, (w, tol)) in enumerate(W.gradients(qs, ks, vs, dos, seen).items()):
            lo, hi = (a, a + n) if name == "dq" else (b, b + m)
            W.assert_close(grads[i][lo:hi], w, tol, f"{name} of sequence {s}")
            assert torch.equal(grads[i][lo:hi], again[i][lo:hi])
        a, b = a + n, b + m


def test_window_is_packed_attention_without_one(ctx):
    """A window as long as the sequence hides nothing: the same bits as packed attention's, where one kernel runs both."""
    q, k, v = normal(80, 500, 4, 64).cuda(), normal(81, 500, 2, 64).cuda(), normal(82, 500, 2, 64).cuda()
    cu = offsets([500])
    a = ctx.packed_attention(q, k, v, cu, causal_block=1)
    assert torch.equal(a, ctx.window_attention(q, k, v, cu))
    assert torch.equal(a, ctx.window_attention(q, k, v, cu, window=500))
    assert torch.equal(a, ctx.window_attention(q, k, v, cu, window=2147483647))
    assert torch.equal(a, ctx.window_attention(q, k, v, cu, window=10, sinks=500))


def test_window_rows_outside_are_left(ctx):
    q, k, v, do = (normal(83 + i, 60, 2, 64).cuda() for i in range(4))
    cu = ints([3, 20, 51])                       # rows 0..2 and 51..59 belong to nobody
    out = torch.full_like(q, 7.0)
    lse = torch.full((2, 60), 7.0, device="cuda")
    grads = [torch.full_like(q, 7.0) for _ in range(3)]
    ctx.window_attention(q, k, v, cu, out=out, window=9, sinks=2, lse=lse)
    ctx.window_attention_backward(q, k, v, out, lse, do, cu, None, *grads, window=9, sinks=2)
    for t in (out, *grads, lse.T):
        assert bool((t[:3] == 7).all()) and bool((t[51:] == 7).all()) and not bool((t[3:51] == 7).all(-1).any())


def test_gradient_is_the_difference(ctx):
    """Differences of the 64-bit formula along a direction, against the library's gradients."""
    n, dim, mask = 40, 64, W.sees(40, 40, 1, 9, 3)
    q, k, v, do = (normal(90 + i, n, 1, dim) for i in range(4))
    lse = torch.empty(1, n, device="cuda")
    out = ctx.window_attention(q.cuda(), k.cuda(), v.cuda(), window=9, sinks=3, lse=lse)
    grads = [g.cpu().double() for g in ctx.window_attention_backward(q.cuda(), k.cuda(), v.cuda(), out, lse, do.cuda(), window=9, sinks=3)]
    tols = [t for _, t in W.gradients(q, k, v, do, mask).values()]
    value = lambda q, k, v: (W.attention(q, k, v, mask)[0] * do.double()).sum()  # noqa: E731
    for i, (g, tol) in enumerate(zip(grads, tols)):
        along = normal(95 + i, n, 1, dim).double()
        step = 1e-5                               # in 64 bits: 1e-16 / step + step^2 is below 1e-10 of the value
        at = [[t.double() + (sign * step * along if j == i else 0) for j, t in enumerate((q, k, v))] for sign in (1, -1)]
        by = float((value(*at[0]) - value(*at[1])) / (2 * step))
        assert abs(by - float((g * along).sum())) <= float((tol * along.abs()).sum()) + 1e-6


def test_together(ctx):
    """A chunk of a prompt as it is served, layer by layer: norm and positions, into the pages, attention; and token
    by token behind it; the same as the whole prompt at once."""
    n, heads, kv_heads, d, page, window, sinks = 300, 4, 2, 128, 16, 90, 5
    x = [normal(110 + i, n, h, d).cuda() for i, h in enumerate((heads, kv_heads, kv_heads))]
    w = [(1 + 0.2 * normal(113 + i, d, dtype=F32)).cuda() for i in range(2)]
    pos = torch.arange(n, dtype=torch.int32, device="cuda").view(1, n)
    q, k = ctx.norm_rotate(x[:2], w, axis_dims=(d,), positions=pos)
    whole = ctx.window_attention(q, k, x[2], window=window, sinks=sinks)
    pages = new_pages(ctx, 40, page, kv_heads, d)
    table = random_table(9, 1, 19, 40).cuda()
    at = 0
    for step in (200, 97, 1, 1, 1):
        rows = slice(at, at + step)
        cq, ck = ctx.norm_rotate([t[rows] for t in x[:2]], w, axis_dims=(d,), positions=pos[:, rows].contiguous())
        assert torch.equal(cq, q[rows]) and torch.equal(ck, k[rows])
        ctx.paged_append(pages, table, ck, x[2][rows], ints([at]))
        at += step
        out = ctx.paged_attention(pages, table, cq, ints([at]), window=window, sinks=sinks)
        want, mag, _, _ = W.attention(q.cpu()[:at], k.cpu()[:at], x[2].cpu()[:at], W.sees(at, at, 1, window, sinks))
        W.assert_attention(out, want[rows], mag[rows], f"{step} tokens")
        W.assert_attention(whole[rows], want[rows], mag[rows], "whole")
        # pages that the window has passed are given away
        for p in range(19):
            if p * page >= sinks and (p + 1) * page <= at + 1 - window and int(table[0, p]) >= 0:
                pages.k[int(table[0, p])] = math.nan
                table[0, p] = -1


# --- the kernels for long key ranges ---------------------------------------------------------------

LONG = [
    # kv heads, group, queries, keys, page
    (2, 1, [1700], None, 64),
    (1, 4, [130, 500], [2100, 1900], 16),
    (12, 1, [2600], None, 256),                  # 252 units
    (1, 2, [300, 1], [1600, 3000], 32),
]
LONG_MASKS = [(0, 0, 0), (1, 0, 0), (1, 700, 0), (1, 1000, 130), (1, 64, 1300), (300, 600, 300), (128, 512, 64), (500, 500, 0), (1, 1, 900)]


@pytest.mark.parametrize("mask", LONG_MASKS, ids=lambda m: "block%d_window%d_sinks%d" % m)
@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_sequences_of_128_dims(ctx, case, mask):
    kv_heads, group, queries, keys, page = LONG[case]
    block, window, sinks = mask
    lengths, heads, d = keys or queries, kv_heads * group, 128
    q, k, v = (normal(200 + i, sum(n), h, d) for i, (n, h) in enumerate(((queries, heads), (lengths, kv_heads), (lengths, kv_heads))))
    kw = dict(causal_block=block, window=window, sinks=sinks)
    lse = torch.full((heads, sum(queries)), math.nan, device="cuda")
    packed = ctx.window_attention(spaced(q), spaced(k), spaced(v), offsets(queries), offsets(lengths) if keys else None, lse=lse, **kw)
    cut = torch.tensor([0] + lengths).cumsum(0).tolist()
    parts = [[t[cut[s]:cut[s + 1]] for s in range(len(lengths))] for t in (k, v)]
    pages, table = fill_pages(ctx, *parts, lengths, page, 8)
    paged = ctx.paged_attention(pages, table, q.cuda(), ints(lengths), offsets(queries), **kw)
    at = 0
    for s, (n, m) in enumerate(zip(queries, lengths)):
        # some heads of the many
        some = list(range(0, heads, max(1, heads // 3)))
        for h in some:
            out, mag, logs, _ = W.attention(q[at:at + n, h:h + 1], parts[0][s][:, h // group:h // group + 1],
                                            parts[1][s][:, h // group:h // group + 1], W.sees(n, m, block, window, sinks))
            W.assert_attention(packed[at:at + n, h:h + 1], out, mag, f"packed {s} {h}")
            W.assert_attention(paged[at:at + n, h:h + 1], out, mag, f"paged {s} {h}")
            got = lse[h, at:at + n].cpu().double()
            assert torch.equal(torch.isinf(got), torch.isinf(logs[0]))
            assert bool((torch.nan_to_num(got - logs[0], nan=0.0).abs() <= 2.0 ** -8 * 1.02).all())
        at += n


@pytest.mark.parametrize("mask", [(1, 0, 0), (1, 1000, 130), (300, 600, 300)], ids=lambda m: "block%d_window%d_sinks%d" % m)
def test_long_sequences_with_large_logits_and_absent_pages(ctx, mask):
    """Units whose fixed softmax offset does not stand run again with a running maximum, and so do those with a page
    that is gone."""
    block, window, sinks = mask
    n, m, d = 400, 2300, 128
    seen = W.sees(n, m, block, window, sinks)
    kw = dict(causal_block=block, window=window, sinks=sinks)
    for spread in (1.0, 40.0):
        q, k, v = normal(210, n, 4, d, spread=spread), normal(211, m, 4, d, spread=spread), normal(212, m, 4, d)
        out, mag, _, _ = W.attention(q, k, v, seen)
        W.assert_attention(ctx.window_attention(q.cuda(), k.cuda(), v.cuda(), None, offsets([m]), **kw), out, mag, "packed")
        pages, table = fill_pages(ctx, [k], [v], [m], 16, 8)
        W.assert_attention(ctx.paged_attention(pages, table, q.cuda(), ints([m]), **kw), out, mag, "paged")
    gone = [(0, p) for p in (0, 3, 70, 121, 143)]
    pages, table = fill_pages(ctx, [k], [v], [m], 16, 8, gone)
    for _, p in gone:
        seen[:, p * 16:(p + 1) * 16] = False
    out, mag, _, _ = W.attention(q, k, v, seen)
    W.assert_attention(ctx.paged_attention(pages, table, q.cuda(), ints([m]), **kw), out, mag, "absent")


@pytest.mark.parametrize("page", [16, 32, 64])
def test_pages_that_the_window_has_passed(ctx, page):
    """A chunk whose window begins inside a tile and a page: giving the pages before it away changes no bit."""
    n, window, sinks, heads = 300, 1000, 40, 2
    lengths = [2301, 1777, 3010]
    k, v = ([normal(220 + s + o, m, heads, 128) for s, m in enumerate(lengths)] for o in (0, 10))
    q = normal(240, 3 * n, 2 * heads, 128).cuda()
    pages, table = fill_pages(ctx, k, v, lengths, page, 8)
    kw = dict(causal_block=1, window=window, sinks=sinks)
    whole = ctx.paged_attention(pages, table, q, ints(lengths), **kw)
    for s, m in enumerate(lengths):
        for p in range(-(-m // page)):
            if p * page >= sinks and (p + 1) * page <= m - n + 1 - window:
                pages.k[int(table[s, p])] = math.nan
                pages.v[int(table[s, p])] = math.nan
                table[s, p] = -1
    assert int((table < 0).sum()) > 3 * 900 // page
    assert torch.equal(ctx.paged_attention(pages, table, q, ints(lengths), **kw), whole)
    for s, m in enumerate(lengths):
        out, mag, _, _ = W.attention(q[s * n:(s + 1) * n].cpu(), k[s], v[s], W.sees(n, m, 1, window, sinks))
        W.assert_attention(whole[s * n:(s + 1) * n], out, mag, f"sequence {s}")
