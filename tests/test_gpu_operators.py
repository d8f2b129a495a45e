"""Rotary positions, attention over packed sequences, and the 4-bit cache with its attention, on
the GPU against the plain 64-bit forms of tests/operators_ref.py."""
import math

import numpy as np
import pytest

import operators_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx(hc):
    c = hc.Context(hc.make_config(n_layers=1), 0)
    yield c
    c.close()


def normal(seed, *shape, dtype=BF, spread=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * spread).to(dtype)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lengths):
    return ints([0] + np.cumsum(lengths).tolist())


def spaced(t, pad=8):
    """The same values on the device in memory with gaps: heads and tokens further apart."""
    n, h, d = t.shape
    big = torch.full((n + 1, h + 1, d + pad), 7.0, dtype=t.dtype, device="cuda")
    view = big[:n, :h, :d]
    view.copy_(t)
    return view


# --- rotary positions ------------------------------------------------------------------------

ROTATE = [
    # tokens, heads, dim, axis_dims, halves, joint, inverse, input, output, far
    (1, 1, 64, (64,), False, False, False, BF, BF, 1 << 20),
    (1, 12, 128, (44, 42, 42), False, False, False, BF, BF, 0),
    (130, 3, 128, (44, 42, 42), False, False, True, BF, F32, 0),
    (77, 5, 64, (24, 20, 20), True, True, False, BF, BF, 0),
    (1000, 2, 128, (16, 56, 56), True, False, False, F32, F32, 2147483647),
    (33, 4, 96, (16, 16, 16), False, True, True, F32, F32, 1 << 20),      # dims behind the rotated ones
    (33, 4, 96, (16, 16, 16), True, False, False, F32, BF, 1000),
    (9, 7, 256, (64, 64, 64, 64), True, True, False, F32, F32, 5000),
    (9, 7, 256, (250, 0, 4, 2), False, False, True, F32, F32, 5000),
    (5, 1, 16, (6, 4, 6), True, False, False, F32, F32, 99),
    (4099, 2, 128, (64, 64), False, False, False, BF, BF, 1 << 30),
]


@pytest.mark.parametrize("case", ROTATE, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}_{len(c[3])}ax")
def test_rotate(ctx, case):
    n, heads, d, axes, halves, joint, inverse, xt, ot, far = case
    x = normal(1, n, heads, d, dtype=xt)
    rot = sum(axes)
    if rot < d:
        x[..., rot:] = normal(2, n, heads, d - rot, dtype=xt)
        x[0, 0, rot] = math.nan                  # copied, and reaches nothing else
        x[0, 0, rot + 1] = -math.inf
    if far:
        pos = torch.from_numpy(np.random.default_rng(3).integers(-far, far, (len(axes), n), dtype=np.int64))
        kw = dict(positions=pos.to(torch.int32).cuda())
    else:
        pos = R.grid_positions(n, 7, 9, 41)
        kw = dict(grid=(7, 9), frame0=41)
    ref = R.rotate(x, pos, axes, 1e4, halves, joint, inverse)
    out = torch.full((heads, n, d), math.nan, dtype=ot, device="cuda").transpose(0, 1)      # head-major
    ctx.rotate(spaced(x), out, axis_dims=axes, halves=halves, joint=joint, inverse=inverse, **kw)
    got = out.cpu().double()
    if rot < d:
        same = x[..., rot:].to(ot)
        assert torch.equal(torch.nan_to_num(got[..., rot:], nan=123.0), torch.nan_to_num(same.double(), nan=123.0))
    # cos and sin: 8.5e-8 of the instruction, 2^-25 of a turn; two products and a sum in 32 bits;
    # angles in 64 bits here and there: j + 3 roundings of position * freq_j, and freq_j (j + 3) < 4
    a = x[..., :rot].double().abs()
    if halves:
        size = (a[..., :rot // 2] + a[..., rot // 2:]).repeat(1, 1, 2)
    else:
        size = (a[..., 0::2] + a[..., 1::2]).repeat_interleave(2, -1)
    tol = size * (8.5e-8 + 2 * math.pi * 2.0 ** -25 + 3 * 2.0 ** -24 + far * 2.0 ** -51) + ref[..., :rot].abs() * torch.finfo(ot).eps / 2
    err = (got - ref)[..., :rot].abs()
    print(f"max err {float(err.max()):.3e}", flush=True)
    assert bool((err <= tol).all())


@pytest.mark.parametrize("n", [1, 63, 2000])
@pytest.mark.parametrize("halves", [False, True])
def test_rotate_pair_in_place(ctx, n, halves):
    q, k = normal(4, n, 12, 128), normal(5, n, 3, 128)
    pos = R.grid_positions(n, 30, 52, 0)
    want = [R.rotate(t, pos, (44, 42, 42), halves=halves) for t in (q, k)]
    dq, dk = q.cuda(), spaced(k)
    got = ctx.rotate((dq, dk), (dq, dk), axis_dims=(44, 42, 42), halves=halves)       # the context's grid
    assert got[0] is dq and got[1] is dk
    for t, w, x in ((dq, want[0], q), (dk, want[1], k)):
        err = (t.cpu().double() - w).abs()
        assert bool((err <= 2.0 ** -8 * w.abs() + 1e-6 * 10).all())


def test_rotate_inverse_is_the_gradient(ctx):
    n, heads, d, axes = 50, 3, 64, (24, 20, 20)
    x, g = normal(6, n, heads, d, dtype=F32).cuda(), normal(7, n, heads, d, dtype=F32).cuda()
    kw = dict(axis_dims=axes, grid=(5, 6), frame0=3)
    back = ctx.rotate(g, inverse=True, **kw)
    # the map is linear, so a difference over any step is its derivative
    step = normal(8, n, heads, d, dtype=F32).cuda()
    along = ((ctx.rotate(x + step, **kw).double() - ctx.rotate(x, **kw).double()) * g.double()).sum()
    assert float(along) == pytest.approx(float((back.double() * step.double()).sum()), rel=1e-4)
    again = ctx.rotate(ctx.rotate(x, **kw), inverse=True, **kw)
    assert float((again - x).abs().max()) < 1e-5


# --- the 4-bit cache --------------------------------------------------------------------------

def same_values(got, want):
    got, want = got.cpu().double(), want.double()
    return bool((torch.isnan(got) == torch.isnan(want)).all()) and \
        bool((torch.nan_to_num(got) == torch.nan_to_num(want)).all())


@pytest.mark.parametrize("seqs,lengths,heads,dim,capacity", [
    (1, [1], 1, 128, 1), (1, [65], 2, 64, 65), (3, [0, 17, 130], 3, 128, 200), (4, [1, 1, 1, 1], 8, 64, 64),
    (2, [64, 64], 1, 128, 64), (70, [3] * 70, 2, 64, 40)])
def test_qcache_round_trip(ctx, seqs, lengths, heads, dim, capacity):
    total = sum(lengths)
    k, v = normal(10, total, heads, dim, spread=3.0), normal(11, total, heads, dim, spread=0.01)
    cache = ctx.qcache(seqs, heads, dim, capacity)
    cache.data.fill_(255)                        # what is not written is not read
    start = ints([min(i % 5, capacity - n) for i, n in enumerate(lengths)])
    cu = offsets(lengths) if len(set(lengths)) > 1 else None
    ctx.qcache_append(cache, spaced(k), v.cuda(), start, cu_seqlens=cu)
    ko, vo = spaced(torch.zeros_like(k)), torch.zeros_like(v, device="cuda")
    ctx.qcache_read(cache, ko, vo, start, cu_seqlens=cu)
    assert same_values(ko, R.stored(k)) and same_values(vo, R.stored(v))


def test_qcache_values_at_their_borders(ctx):
    """Every bf16 magnitude pattern near a rounding border, at several scales, subnormals, the
    largest finite values, and groups that are not finite."""
    rows = []
    for e in (-133, -127, -126, -125, -124, -30, 0, 60, 124, 125, 126, 127):
        for top in (1.0, 1.5, 1.75, 1.7578125, 1.9921875):
            steps = torch.arange(31) / 16.0 * top * 0.515625
            rows.append(torch.cat([torch.ldexp(torch.tensor([top]), torch.tensor(e)).double(),
                                   torch.ldexp(steps.double(), torch.tensor(e))]))
    for bad in (math.inf, -math.inf, math.nan):
        r = torch.ones(32, dtype=torch.float64)
        r[5] = bad
        rows.append(r)
    x = torch.stack(rows)
    x[:, 1::2] *= -1
    x = torch.cat([x, torch.zeros(-x.shape[0] % 4, 32, dtype=torch.float64)]).to(BF).reshape(-1, 1, 128)
    n = x.shape[0]
    cache = ctx.qcache(1, 1, 128, n)
    ctx.qcache_append(cache, x.cuda(), x.flip(0).contiguous().cuda(), ints([0]))
    k, v = torch.zeros(n, 1, 128, dtype=BF, device="cuda"), torch.zeros(n, 1, 128, dtype=BF, device="cuda")
    ctx.qcache_read(cache, k, v, ints([0]))
    want = R.stored(x)
    assert same_values(k, want) and same_values(v, want.flip(0))


def test_qcache_overwrites_and_leaves_the_rest(ctx):
    heads, dim, cap = 2, 128, 100
    a, b = normal(12, cap, heads, dim), normal(13, 7, heads, dim)
    cache = ctx.qcache(1, heads, dim, cap)
    ctx.qcache_append(cache, a.cuda(), a.cuda(), ints([0]))
    ctx.qcache_append(cache, b.cuda(), b.cuda(), ints([61]))
    want = R.stored(a)
    want[61:68] = R.stored(b)
    k, v = torch.zeros_like(a, device="cuda"), torch.zeros_like(a, device="cuda")
    ctx.qcache_read(cache, k, v, ints([0]))
    assert same_values(k, want) and same_values(v, want)


def test_qcache_slots_out_of_range_are_left_alone(ctx):
    heads, dim, cap = 1, 64, 70
    cache = ctx.qcache(2, heads, dim, cap)
    base = normal(14, 2 * cap, heads, dim)
    ctx.qcache_append(cache, base.cuda(), base.cuda(), ints([0, 0]))
    new = normal(15, 12, heads, dim)
    # sequence 0: slots -3 .. 2, sequence 1: slots 67 .. 72; rows 10 and 11 belong to none
    ctx.qcache_append(cache, new.cuda(), new.cuda(), ints([-3, 67]), cu_seqlens=ints([0, 5, 10]))
    want = R.stored(base)
    put = R.stored(new)
    want[0:2] = put[3:5]
    want[cap + 67:cap + 70] = put[5:8]
    k, v = torch.zeros_like(base, device="cuda"), torch.zeros_like(base, device="cuda")
    ctx.qcache_read(cache, k, v, ints([0, 0]))
    assert same_values(k, want) and same_values(v, want)
    k.fill_(5.0)
    ctx.qcache_read(cache, k[:12], v[:12], ints([-3, 67]), cu_seqlens=ints([0, 5, 10]))
    got = k[:12].cpu().double()
    assert bool((got[:3] == 5.0).all()) and bool((got[8:] == 5.0).all())
    assert same_values(k[3:8], torch.cat([want[0:2], want[cap + 67:cap + 70]]))


# --- attention over packed sequences -----------------------------------------------------------

PACKED = [
    # query lengths, key lengths (None: the same), key heads, group, dim, block
    ([1], None, 1, 1, 64, 1),
    ([1], None, 2, 3, 128, 0),
    ([77], None, 12, 1, 64, 1),
    ([64, 65], None, 2, 1, 128, 1),
    ([1, 0, 129, 5, 300], None, 2, 4, 128, 1),
    ([200, 3, 0, 77], None, 3, 5, 64, 0),
    ([513], None, 1, 7, 128, 96),
    ([130, 260], None, 2, 2, 64, 65),
    ([10, 128, 3], [300, 1, 0], 2, 2, 128, 0),
    ([10, 128, 3], [300, 100, 0], 2, 2, 128, 1),      # more queries than keys: the first see nothing
    ([70, 20], [65, 500], 1, 3, 64, 7),
    ([1500], None, 1, 1, 128, 1),
    ([3], [5000], 2, 1, 128, 1),                      # few rows, many keys: split
    ([40, 1], [2100, 3000], 1, 4, 64, 0),
    ([2] * 150, None, 1, 2, 64, 1),
]


def packed_case(ctx, case, seed=20, q_spread=1.0, v_shift=0.0):
    nq, nk, kv_heads, group, d, block = case
    nk_ = nq if nk is None else nk
    q = normal(seed, sum(nq), kv_heads * group, d, spread=q_spread)
    k, v = normal(seed + 1, sum(nk_), kv_heads, d), normal(seed + 2, sum(nk_), kv_heads, d) + v_shift
    out = torch.full((sum(nq) + 3, kv_heads * group, d), 9.0, dtype=BF, device="cuda")
    qd = torch.cat([q, normal(seed + 3, 3, *q.shape[1:])]).cuda()      # rows behind the last sequence
    kd, vd = spaced(k), spaced(v)
    if nk is None:                               # (the keys of those rows)
        kd = spaced(torch.cat([k, torch.full((3, *k.shape[1:]), math.nan, dtype=BF)]))
        vd = spaced(torch.cat([v, torch.full((3, *k.shape[1:]), math.nan, dtype=BF)]))
    ctx.packed_attention(qd, kd, vd, offsets(nq), None if nk is None else offsets(nk), out=out, causal_block=block)
    assert bool((out[sum(nq):] == 9.0).all())
    ref, mag = [], []
    a = b = 0
    for n, m in zip(nq, nk_):
        r = R.attention(q[a:a + n], k[b:b + m], v[b:b + m], block)
        ref.append(r[0])
        mag.append(r[1])
        a, b = a + n, b + m
    R.assert_attention(out[:sum(nq)], torch.cat(ref), torch.cat(mag), str(case))
    return out


@pytest.mark.parametrize("case", PACKED, ids=lambda c: f"q{len(c[0])}x{max(c[0])}_h{c[2]}x{c[3]}_d{c[4]}_b{c[5]}")
def test_packed_attention(ctx, case):
    packed_case(ctx, case)


# Long key ranges: every path of the kernels for 128-dim heads (the written-out steps, the look at the row
# sums, tiles that not all rows see whole, ranges that share units evenly), against 64 bits on the GPU.
LONG = [
    # queries, keys, key heads, group, block
    (1000, 5000, 4, 1, 0),
    (2000, 2000, 8, 2, 1),
    (1500, 3500, 6, 3, 700),
    (4200, 8300, 9, 1, 0),           # 297 units on 512 places
    (8000, 8200, 9, 1, 0),           # 567 units
    (4096, 8192, 12, 1, 0),          # whole units only, 384 of them
    (640, 9000, 3, 1, 1),
]


def long_reference(q, k, v, block, scale=None):
    n, heads, d = q.shape
    m, group = k.shape[0], heads // k.shape[1]
    count = torch.tensor(R.seen(n, m, block), device="cuda").unsqueeze(1)
    hidden = torch.arange(m, device="cuda") >= count
    out, mag = [], []
    for h in range(heads):
        p = q[:, h].double() @ k[:, h // group].double().T * (scale if scale else d ** -0.5)
        p = torch.softmax(p.masked_fill_(hidden, -math.inf), -1)
        w = v[:, h // group].double()
        out.append(p @ w)
        mag.append(p @ w.abs())
    return torch.stack(out, 1).cpu(), torch.stack(mag, 1).cpu()


@pytest.mark.parametrize("spread", [1.0, 40.0])
@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("case", LONG, ids=lambda c: "x".join(map(str, c)))
def test_long_key_ranges(ctx, case, cached, spread):
    n, m, kv_heads, group, block = case
    q = normal(80, n, kv_heads * group, 128, spread=spread).cuda()
    k, v = normal(81, m, kv_heads, 128).cuda(), normal(82, m, kv_heads, 128).cuda()
    if cached:
        cache = ctx.qcache(1, kv_heads, 128, m + 100)
        cache.data.fill_(255)
        ctx.qcache_append(cache, k, v, ints([0]))
        ctx.qcache_read(cache, k, v, ints([0]))
        got = ctx.qcache_attention(cache, q, ints([m]), ints([0, n]), causal_block=block)
    else:
        got = ctx.packed_attention(q, k, v, ints([0, n]), ints([0, m]), causal_block=block)
    R.assert_attention(got, *long_reference(q, k, v, block), str(case))


def test_even_shares_with_fewer_rows_and_keys_than_planned(ctx):
    """Offsets and lengths on the device that name less than the tensors hold."""
    q, k, v = (normal(83 + i, n, 9, 128).cuda() for i, n in enumerate((4200, 8300, 8300)))
    for nq, nk in ((3000, 8300), (4200, 900), (130, 65), (4200, 0)):
        out = torch.full_like(q, 9.0)
        ctx.packed_attention(q, k, v, ints([0, nq]), ints([0, nk]), out=out)
        assert bool((out[nq:] == 9.0).all())
        if nk:
            R.assert_attention(out[:nq], *long_reference(q[:nq], k[:nk], v[:nk], 0), f"{nq} {nk}")
        else:
            assert bool((out == 0).all())


@pytest.mark.parametrize("d", [64, 128])
def test_many_sequences_in_any_order(ctx, d):
    """More sequences than are ranked, and fewer, with lengths in no order."""
    for n_seqs in (20, 90):
        rng = np.random.default_rng(n_seqs)
        nq, nk = rng.integers(0, 200, n_seqs).tolist(), rng.integers(0, 300, n_seqs).tolist()
        packed_case(ctx, (nq, nk, 2, 2, d, 1), seed=90)


@pytest.mark.parametrize("spread", [1e-3, 40.0, 1000.0])
@pytest.mark.parametrize("d", [64, 128])
def test_packed_attention_logit_range(ctx, spread, d):
    """Logits that are all alike, and ones that leave a single key per row."""
    packed_case(ctx, ([300, 140], None, 2, 2, d, 1), seed=30, q_spread=spread)


def test_packed_equal_parts_and_scale(ctx):
    q, k, v = normal(40, 96, 4, 64), normal(41, 96, 4, 64), normal(42, 96, 4, 64)
    got = ctx.packed_attention(q.cuda(), k.cuda(), v.cuda(), n_seqs=3, causal_block=1, softmax_scale=0.3)
    for s in range(3):
        at = slice(32 * s, 32 * s + 32)
        R.assert_attention(got[at], *R.attention(q[at], k[at], v[at], 1, 0.3))


def test_packed_head_major_and_shared_rows(ctx):
    """Head-major tensors, and one key head expanded to several without a copy."""
    q, k, v = normal(43, 6, 200, 128), normal(44, 1, 200, 128), normal(45, 1, 200, 128)
    qd = q.cuda().transpose(0, 1)
    kd, vd = (t.cuda().transpose(0, 1).expand(200, 3, 128) for t in (k, v))
    out = torch.empty(6, 200, 128, dtype=BF, device="cuda").transpose(0, 1)
    ctx.packed_attention(qd, kd, vd, out=out, causal_block=1)
    R.assert_attention(out, *R.attention(q.transpose(0, 1), k.transpose(0, 1), v.transpose(0, 1), 1))


def test_strides_of_axes_of_length_one(ctx):
    """One token, one key and one head cut out of larger tensors at any stride."""
    q = normal(60, 3, 5, 68).cuda().as_strided((1, 1, 64), (3, 5, 1))
    k = normal(61, 3, 5, 68).cuda().as_strided((1, 1, 64), (7, 1, 1))
    out = torch.zeros(1, 1, 64, dtype=BF, device="cuda").as_strided((1, 1, 64), (1, 1, 1))
    ctx.packed_attention(q, k, k, out=out, causal_block=1)
    assert torch.equal(out, k)
    turned = ctx.rotate(q, axis_dims=(24, 20, 20), grid=(1, 1), frame0=5)
    ref = R.rotate(q.cpu(), torch.tensor([[5], [0], [0]]), (24, 20, 20))
    assert bool(((turned.cpu().double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-5).all())


def test_packed_bad_values_stay_in_their_sequence(ctx):
    nq = [50, 40, 60]
    q, k, v = normal(46, 150, 2, 128), normal(47, 150, 2, 128), normal(48, 150, 2, 128)
    k[50:90], v[50:90] = math.nan, math.inf
    got = ctx.packed_attention(q.cuda(), k.cuda(), v.cuda(), offsets(nq), causal_block=1)
    for at in (slice(0, 50), slice(90, 150)):
        R.assert_attention(got[at], *R.attention(q[at], k[at], v[at], 1))
    assert not torch.isfinite(got[50:90]).any()


def test_packed_bad_values_stay_in_their_sequence_over_long_ranges(ctx):
    """The same where the written-out steps run, with sequences that share neither rows nor tiles."""
    n = 2100
    q, k, v = (normal(49 + i, 2 * n, 2, 128).cuda() for i in range(3))
    k[n:], v[n:] = math.nan, math.nan
    got = ctx.packed_attention(q, k, v, ints([0, n, 2 * n]), causal_block=0)
    R.assert_attention(got[:n], *long_reference(q[:n], k[:n], v[:n], 0))
    assert bool(torch.isnan(got[n:]).all())


def test_two_graphs_with_workspaces_of_their_own(ctx):
    """Two captured calls that need room for partial results, replayed at the same time on two streams."""
    n, m = 5, 6000
    sides = []
    for s in range(2):
        q, k, v = normal(52 + s, n, 4, 128).cuda(), normal(54 + s, m, 2, 128).cuda(), normal(56 + s, m, 2, 128).cuda()
        cu = (ints([0, n]), ints([0, m]))
        out = torch.zeros_like(q)
        work = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
        call = lambda q=q, k=k, v=v, cu=cu, out=out, work=work: ctx.packed_attention(q, k, v, *cu, out=out, causal_block=1, workspace=work)  # noqa: E731
        call()
        torch.cuda.synchronize()
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        sides.append((graph, out, want, torch.cuda.Stream(), call))     # (the call holds its tensors)
    for _ in range(5):
        for _, out, _, _, _ in sides:
            out.zero_()
        torch.cuda.synchronize()
        for graph, _, _, stream, _ in sides:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, out, want, _, _ in sides:
            assert torch.equal(out, want)


def test_refusals_through_the_binding(ctx, hc):
    q = normal(58, 8, 4, 64).cuda()
    cu = ints([0, 8])
    with pytest.raises(ValueError, match="bfloat16"):
        ctx.packed_attention(q.float(), q, q, cu)
    with pytest.raises(hc.HeadCastError, match="multiple of n_kv_heads"):
        ctx.packed_attention(q, q[:, :3], q[:, :3], cu)
    with pytest.raises(hc.HeadCastError, match="strides"):
        odd = torch.zeros(8, 4, 68, dtype=BF, device="cuda")[..., :64]
        ctx.packed_attention(odd, q, q, cu)
    with pytest.raises(hc.HeadCastError, match="rows overlap"):
        ctx.packed_attention(q, q, q, cu, out=torch.zeros(1, 4, 64, dtype=BF, device="cuda").expand(8, 4, 64))
    with pytest.raises(hc.HeadCastError, match="workspace"):
        k = normal(59, 6000, 1, 64).cuda()
        ctx.packed_attention(q[:2, :1], k, k, ints([0, 2]), ints([0, 6000]),
                             workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="int32"):
        ctx.packed_attention(q, q, q, cu.long())
    with pytest.raises(hc.HeadCastError, match="axis_dims"):
        ctx.rotate(q, axis_dims=(24, 20, 10))
    cache = ctx.qcache(1, 4, 64, 10)
    with pytest.raises(ValueError, match="start"):
        ctx.qcache_append(cache, q, q, ints([0, 0]))
    with pytest.raises(ValueError, match="expected shape"):
        ctx.qcache_append(cache, q[:, :2], q, ints([0]))


# --- attention over the 4-bit cache --------------------------------------------------------------

CACHED = [
    # query lengths, key counts, capacity, key heads, group, dim, block
    ([1], [1], 1, 1, 1, 64, 1),
    ([1], [65], 65, 2, 1, 128, 0),
    ([1, 1, 1], [0, 64, 200], 200, 2, 7, 64, 1),
    ([1, 1], [5000, 129], 5000, 1, 4, 128, 1),
    ([1] * 70, list(range(1, 71)), 90, 2, 8, 128, 1),
    ([3, 0, 5], [100, 50, 3], 128, 2, 2, 128, 1),         # the last: more queries than keys
    ([33], [700], 700, 1, 1, 64, 1),
    ([300, 20], [1000, 333], 1024, 2, 3, 128, 1),
    ([128], [640], 640, 3, 1, 64, 0),
    ([200], [600], 600, 1, 2, 128, 50),
    ([9, 250, 1], [9, 250, 1], 256, 2, 1, 64, 1),
    ([2], [3000], 3000, 1, 16, 64, 1),
]


def cached_inputs(ctx, case, seed=60):
    nq, nk, cap, kv_heads, group, d, block = case
    k, v = normal(seed, len(nk) * cap, kv_heads, d), normal(seed + 1, len(nk) * cap, kv_heads, d)
    cache = ctx.qcache(len(nk), kv_heads, d, cap)
    cache.data.fill_(255)                        # slots never written read as NaN
    lengths = offsets(nk)
    rows = torch.cat([torch.arange(m) + s * cap for s, m in enumerate(nk)])
    ctx.qcache_append(cache, k[rows].cuda(), v[rows].cuda(), ints([0] * len(nk)), cu_seqlens=lengths)
    return cache, normal(seed + 2, sum(nq), kv_heads * group, d), k, v


def cached_reference(case, q, k, v):
    nq, nk, cap, kv_heads, group, d, block = case
    ref, mag, a = [], [], 0
    for s, (n, m) in enumerate(zip(nq, nk)):
        r = R.attention(q[a:a + n], R.stored(k[s * cap:s * cap + m]), R.stored(v[s * cap:s * cap + m]), block)
        ref.append(r[0])
        mag.append(r[1])
        a += n
    return torch.cat(ref), torch.cat(mag)


@pytest.mark.parametrize("case", CACHED, ids=lambda c: f"q{len(c[0])}x{max(c[0])}_k{max(c[1])}_h{c[3]}x{c[4]}_d{c[5]}_b{c[6]}")
def test_qcache_attention(ctx, case):
    nq, nk = case[0], case[1]
    cache, q, k, v = cached_inputs(ctx, case)
    out = torch.full((sum(nq) + 2, *q.shape[1:]), 9.0, dtype=BF, device="cuda")
    qd = torch.cat([q, q[:1], q[:1]])
    ctx.qcache_attention(cache, spaced(qd), ints(nk), offsets(nq), out=out, causal_block=case[6])
    assert bool((out[sum(nq):] == 9.0).all())
    R.assert_attention(out[:sum(nq)], *cached_reference(case, q, k, v), str(case))


def test_qcache_attention_lengths_are_clamped(ctx):
    case = ([1, 1], [50, 50], 50, 1, 2, 64, 1)
    cache, q, k, v = cached_inputs(ctx, case)
    got = ctx.qcache_attention(cache, q.cuda(), ints([1000, -4]), causal_block=1)
    ref, mag = cached_reference(case, q, k, v)
    R.assert_attention(got[:1], ref[:1], mag[:1])
    assert bool((got[1:] == 0).all())


def test_qcache_attention_hint_changes_nothing_but_rounding(ctx):
    case = ([1, 2, 4], [3000, 100, 2000], 3000, 2, 4, 128, 1)
    cache, q, k, v = cached_inputs(ctx, case)
    ref, mag = cached_reference(case, q, k, v)
    for hint in (0, 1, 500, 3000, 1 << 30):
        got = ctx.qcache_attention(cache, q.cuda(), ints(case[1]), offsets(case[0]), causal_block=1, max_kv=hint)
        R.assert_attention(got, ref, mag, f"max_kv {hint}")


def test_qcache_attention_group_that_is_not_finite(ctx):
    case = ([2, 2], [100, 100], 100, 1, 1, 128, 0)
    cache, q, k, v = cached_inputs(ctx, case)
    bad = torch.full((1, 1, 128), math.inf, dtype=BF, device="cuda")
    good = torch.zeros(1, 1, 128, dtype=BF, device="cuda")
    ctx.qcache_append(cache, good, bad, ints([0, 70]), cu_seqlens=ints([0, 0, 1]))
    got = ctx.qcache_attention(cache, q.cuda(), ints([100, 100]), causal_block=0)
    ref, mag = cached_reference(case, q, k, v)
    R.assert_attention(got[:2], ref[:2], mag[:2])
    assert bool(torch.isnan(got[2:]).all())


# --- together, as a step uses them -----------------------------------------------------------------

def block_step(ctx, state):
    """A block's step: rotate, store the keys and values in the window, attend over it."""
    c = ctx
    c.rotate((state["q"], state["k"]), (state["qr"], state["kr"]), axis_dims=(44, 42, 42), grid=(8, 10), frame0=6)
    c.qcache_append(state["cache"], state["kr"], state["v"], state["start"])
    c.qcache_attention(state["cache"], state["qr"], state["len"], out=state["o"], causal_block=0,
                       workspace=state["work"])
    c.packed_attention(state["o"], state["tk"], state["tv"], state["cu_q"], state["cu_k"], out=state["o2"],
                       workspace=state["work2"])


def step_state(ctx, seed):
    n, heads = 160, 3
    s = {x: normal(seed + i, n, heads, 128).cuda() for i, x in enumerate("qkv")}
    s["qr"], s["kr"], s["o"], s["o2"] = (torch.zeros(n, heads, 128, dtype=BF, device="cuda") for _ in range(4))
    s["tk"], s["tv"] = normal(seed + 5, 30, heads, 128).cuda(), normal(seed + 6, 30, heads, 128).cuda()
    s["cu_q"], s["cu_k"] = ints([0, n]), ints([0, 30])
    s["cache"] = ctx.qcache(1, heads, 128, 4 * n)
    old = [normal(seed + 7 + i, 2 * n, heads, 128).cuda() for i in range(2)]
    ctx.qcache_append(s["cache"], *old, ints([0]))
    s["start"], s["len"] = ints([2 * n]), ints([3 * n])
    s["work"], s["work2"] = (torch.empty(8 << 20, dtype=torch.uint8, device="cuda") for _ in range(2))
    s["old"] = old
    return s


def step_reference(s):
    pos = R.grid_positions(160, 8, 10, 6)
    qr = s["qr"].cpu()
    for x, r in (("q", "qr"), ("k", "kr")):
        ref = R.rotate(s[x].cpu(), pos, (44, 42, 42))
        assert bool(((s[r].cpu().double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-5).all())
    k, v = (torch.cat([R.stored(s["old"][i].cpu()), R.stored(s[x].cpu())]) for i, x in ((0, "kr"), (1, "v")))
    R.assert_attention(s["o"], *R.attention(qr, k, v, 0), "window")
    R.assert_attention(s["o2"], *R.attention(s["o"].cpu(), s["tk"].cpu(), s["tv"].cpu(), 0), "text")


def test_step_together(ctx):
    s = step_state(ctx, 100)
    block_step(ctx, s)
    step_reference(s)


def test_step_captured_and_replayed(ctx):
    s = step_state(ctx, 200)
    block_step(ctx, s)
    want = s["o2"].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block_step(ctx, s)
    other = step_state(ctx, 300)
    for i in range(4):
        for x in ("qr", "kr", "o", "o2"):
            s[x].zero_()
        graph.replay()
        block_step(ctx, other)                   # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(s["o2"], want), f"replay {i}"
    # lengths and slots are read at replay: one block further
    s["start"].fill_(480)
    s["len"].fill_(640)
    s["old"] = [torch.cat([t, s[x]]) for t, x in zip(s["old"], ("kr", "v"))]
    graph.replay()
    torch.cuda.synchronize()
    step_reference(s)


def test_on_another_stream(ctx):
    s = step_state(ctx, 400)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block_step(ctx, s)
    side.synchronize()
    step_reference(s)


def test_schedule_rotates_its_blocks(hc):
    """The autoregressive schedule on blocks without positions does what it does on rotated ones."""
    from paper_2607_20125_amd import ar_loop
    from synth import inputs as S
    w = S.WORKLOADS["tiny"]
    axes, blocks = (24, 20, 20), w.window_blocks + 2
    data = {(b, i): tuple(normal(1000 + 10 * b + i, 3, w.n_heads, w.block_tokens, w.head_dim)) for b in range(blocks)
            for i in range(2)}
    seen = []
    for rotated in (False, True):
        ctx = hc.Context(hc.config_from_workload(w, n_layers=1), 0)

        def block(layer, b, step):
            q, k, v = (t.cuda() for t in data[b, step])
            if rotated:
                pos = R.grid_positions(w.block_tokens, w.grid_h, w.grid_w, b * w.frames_per_block)
                q, k = (ctx.rotate(t.transpose(0, 1).contiguous(), axis_dims=axes, positions=pos.int().cuda())
                        .transpose(0, 1).contiguous() for t in (q, k))
            return q, k, v

        out = torch.zeros(w.n_heads, w.block_tokens, w.head_dim, device="cuda")
        outs = []
        ar_loop.run(ctx, blocks, block, out, steps=(1000, 500), on_step=lambda *a: outs.append(out.clone()),
                    tables_at_fill=[[0, 1, 2, 3]], classify=False, axis_dims=None if rotated else axes)
        seen.append(torch.stack(outs))
        ctx.close()
    assert torch.isfinite(seen[0]).all() and torch.equal(seen[0], seen[1])


def test_profile_counts(hc):
    c = hc.Context(hc.make_config(n_layers=1), 0)
    s = step_state(c, 500)
    c.profile_enable()
    block_step(c, s)
    assert [c.profile_read(k)[1] for k in (hc.K_ROTATE, hc.K_CACHE, hc.K_SEQUENCE)] == [1, 1, 2]
    c.close()


def test_cache_longer_than_32_bit_offsets(ctx):
    """Codes behind the 2^32nd byte of a cache."""
    cap, heads = 1 << 20, 32                     # 17.4 KB per 64 tokens and head pair: 4.6 GB
    cache = ctx.qcache(1, heads, 128, cap)
    assert cache.data.numel() > 1 << 32
    n = 100
    k, v = normal(70, n, heads, 128), normal(71, n, heads, 128)
    ctx.qcache_append(cache, k.cuda(), v.cuda(), ints([cap - n]))
    ko, vo = torch.zeros_like(k, device="cuda"), torch.zeros_like(v, device="cuda")
    ctx.qcache_read(cache, ko, vo, ints([cap - n]))
    assert same_values(ko, R.stored(k)) and same_values(vo, R.stored(v))
