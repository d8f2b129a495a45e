"""What the attentions over sequences and over the 4-bit cache make of values that are rare: every kernel and
every plan of key ranges, several sequences at once, on the GPU against 64 bits."""
import math

import numpy as np
import pytest

import operators_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx(hc):
    c = hc.Context(hc.make_config(n_layers=1), 0)
    yield c
    c.close()


def normal(seed, *shape, spread=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * spread).to(BF)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lengths):
    return ints([0] + np.cumsum(lengths).tolist())


def parts(x, lengths):
    return torch.split(x, list(lengths))


def reference(q, k, v, block):
    """(output, sum p |v|) of one sequence in 64 bits on the GPU."""
    (n, heads, d), (m, kv_heads, _) = q.shape, k.shape
    out, mag = torch.zeros(n, heads, d, dtype=torch.float64), torch.zeros(n, heads, d, dtype=torch.float64)
    if n == 0 or m == 0:
        return out, mag
    count = torch.tensor(R.seen(n, m, block), device="cuda").unsqueeze(1)
    hidden = torch.arange(m, device="cuda") >= count
    for h in range(heads):
        kh, w = k[:, h // (heads // kv_heads)].double(), v[:, h // (heads // kv_heads)].double()
        p = torch.softmax((q[:, h].double() @ kh.T.contiguous() * d ** -0.5).masked_fill_(hidden, -math.inf), -1)
        p = torch.where(count == 0, 0.0, p)
        out[:, h], mag[:, h] = (p @ w).cpu(), (p @ w.abs()).cpu()
    return out, mag


def attend(ctx, cached, q, k, v, nq, nk, block, capacity=None):
    """The attention of all sequences, and the keys and values that it is of (those that a cache stands for)."""
    out = torch.full_like(q, 9.0)
    if not cached:
        return ctx.packed_attention(q, k, v, offsets(nq), offsets(nk), out=out, causal_block=block), k, v
    cache = ctx.qcache(len(nk), k.shape[1], k.shape[2], capacity or max(nk))
    cache.data.fill_(255)                        # slots never written read as NaN
    start, cu = ints([0] * len(nk)), offsets(nk)
    ctx.qcache_append(cache, k, v, start, cu_seqlens=cu)
    ks, vs = torch.zeros_like(k), torch.zeros_like(v)
    ctx.qcache_read(cache, ks, vs, start, cu_seqlens=cu)
    return ctx.qcache_attention(cache, q, ints(nk), offsets(nq), out=out, causal_block=block), ks, vs


# --- values that are not finite -------------------------------------------------------------------

NOT_FINITE = [
    # cached, queries, keys, key heads, group, dim, capacity: the kernel and its plan
    (True, [2, 2, 1], [100, 90, 30], 2, 2, 64, None),          # few rows, uncut
    (True, [2, 2, 1], [100, 90, 30], 2, 2, 128, None),
    (True, [1, 1, 1], [3000, 4000, 900], 1, 4, 64, None),      # few rows in many ranges
    (True, [1, 1, 1], [3000, 4000, 900], 1, 4, 128, None),
    (True, [1, 1, 1], [700, 600, 500], 8, 2, 128, None),       # few rows in a few ranges
    (True, [100, 70, 90], [200, 300, 100], 2, 2, 64, None),    # waves of 32 rows, uncut
    (True, [100, 70, 90], [200, 300, 100], 2, 2, 128, None),
    (True, [100, 70, 90], [2000, 1900, 1100], 2, 2, 64, None),     # ... cut
    (True, [200, 150, 180], [2000, 1900, 1700], 2, 2, 128, None),  # waves of 64 rows, cut
    (True, [1500, 1400, 1200], [450, 500, 640], 4, 2, 128, None),  # ... uncut
    (True, [100, 70, 90], [6000, 5000, 5500], 1, 1, 64, None),     # many ranges of whole tiles of rows
    (False, [100, 70, 90], [6000, 5000, 5500], 1, 1, 128, None),
    (False, [100, 70, 90], [200, 300, 100], 2, 2, 64, None),
    (False, [100, 70, 90], [200, 300, 100], 2, 2, 128, None),
    (False, [100, 70, 90], [2000, 1900, 1100], 2, 2, 64, None),
    (False, [200, 150, 180], [2000, 1900, 1700], 2, 2, 128, None),
    (False, [1500, 1400, 1200], [450, 500, 640], 4, 2, 128, None),
]


@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("case", NOT_FINITE, ids=lambda c: f"{'cached' if c[0] else 'packed'}_q{c[1][0]}_k{c[2][0]}_d{c[5]}")
def test_values_that_are_not_finite(ctx, case, where):
    """One value of the second sequence that is not finite: a key gives NaN to the rows of its head, a value to its dim
    (its 32 dims in a cache); everything else is as it is without."""
    cached, nq, nk, kv_heads, group, d, capacity = case
    q = normal(1, sum(nq), kv_heads * group, d)
    k, v = normal(2, sum(nk), kv_heads, d), normal(3, sum(nk), kv_heads, d)
    bad = torch.tensor(math.nan if not cached or where == "k" else math.inf, dtype=BF)
    head, dim = kv_heads - 1, 37
    (k if where == "k" else v)[nk[0] + nk[1] // 2, head, dim] = bad
    got, k, v = attend(ctx, cached, q, k, v, nq, nk, 0, capacity)
    spoiled = torch.zeros(sum(nq), kv_heads * group, d, dtype=torch.bool)
    dims = slice(0, d) if where == "k" else slice(32, 64) if cached else slice(dim, dim + 1)
    spoiled[nq[0]:nq[0] + nq[1], head * group:, dims] = True
    got = got.cpu().double()
    assert bool(torch.isnan(got[spoiled]).all())
    k, v = torch.nan_to_num(k, nan=0.0), torch.nan_to_num(v, nan=0.0)
    refs = [reference(*x, 0) for x in zip(parts(q, nq), parts(k, nk), parts(v, nk))]
    out, mag = (torch.cat([r[i] for r in refs]) for i in range(2))
    R.assert_attention(torch.where(spoiled, out, got), out, mag, str(case))


# --- outputs in the queries' place ----------------------------------------------------------------

@pytest.mark.parametrize("case", NOT_FINITE, ids=lambda c: f"{'cached' if c[0] else 'packed'}_q{c[1][0]}_k{c[2][0]}_d{c[5]}")
def test_outputs_over_the_queries(ctx, case):
    cached, nq, nk, kv_heads, group, d, _ = case
    q = normal(11, sum(nq), kv_heads * group, d)
    k, v = normal(12, sum(nk), kv_heads, d), normal(13, sum(nk), kv_heads, d)
    if cached:
        cache = ctx.qcache(len(nk), kv_heads, d, max(nk))
        ctx.qcache_append(cache, k, v, ints([0] * len(nk)), cu_seqlens=offsets(nk))
        call = lambda out: ctx.qcache_attention(cache, q, ints(nk), offsets(nq), out=out, causal_block=1)  # noqa: E731
    else:
        call = lambda out: ctx.packed_attention(q, k, v, offsets(nq), offsets(nk), out=out, causal_block=1)  # noqa: E731
    want = call(None)
    assert call(q) is q and torch.equal(q, want)


# --- large logits -----------------------------------------------------------------------------------

@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("case", NOT_FINITE, ids=lambda c: f"{'cached' if c[0] else 'packed'}_q{c[1][0]}_k{c[2][0]}_d{c[5]}")
def test_logits_close_to_2_to_the_28(ctx, case, sign):
    """Logits of one sign up to 2^27.6 (log2 units) that 32 bits hold exactly, three different ones: a row is the mean of
    the values whose key is best."""
    cached, nq, nk, kv_heads, group, d, _ = case
    q = torch.full((sum(nq), kv_heads * group, d), sign * 2.0 ** 10, dtype=BF, device="cuda")
    level = torch.tensor([9.0, 10.0, 12.0], device="cuda")[torch.arange(sum(nk), device="cuda") * 7 % 11 % 3]
    k = (level * 2.0 ** 10)[:, None, None].expand(-1, kv_heads, d).to(BF).contiguous()
    v = normal(21, sum(nk), kv_heads, d)
    got, k, v = attend(ctx, cached, q, k, v, nq, nk, 0)
    refs = [reference(*x, 0) for x in zip(parts(q, nq), parts(k, nk), parts(v, nk))]
    R.assert_attention(got, *(torch.cat([r[i] for r in refs]) for i in range(2)), str(case))


def test_schedule_rotates_blocks_that_require_gradients(hc):
    """The schedule records none, so a block from a model's projections runs as a detached one does."""
    from paper_2607_20125_amd import ar_loop
    from synth import inputs as S
    w = S.WORKLOADS["tiny"]
    outs = []
    for grad in (False, True):
        c = hc.Context(hc.config_from_workload(w, n_layers=1), 0)
        out = torch.zeros(w.n_heads, w.block_tokens, w.head_dim, device="cuda")

        def block(layer, b, step):
            return tuple(normal(30 + 3 * b + i, w.n_heads, w.block_tokens, w.head_dim).requires_grad_(grad) for i in range(3))

        ar_loop.run(c, 2, block, out, steps=(1000,), classify=False, axis_dims=(24, 20, 20))
        outs.append(out)
        c.close()
    assert torch.isfinite(outs[0]).all() and torch.equal(*outs)


# --- several sequences ------------------------------------------------------------------------------

SEVERAL = [
    # queries, keys, key heads, group, block: 128-dim heads on waves of 64 rows
    ([700, 1300, 65], [1900, 3333, 1601], 2, 3, 1),                       # key ranges
    ([700, 1300, 65], [1900, 3333, 1601], 2, 3, 700),
    ([400, 0, 800], [2000, 1700, 1999], 2, 1, 0),
    ([500, 900], [300, 2901], 1, 2, 1),                                   # the first queries see nothing
    ([100, 300, 700], [0, 2500, 2333], 3, 1, 1),
    ([2000, 1111, 300, 1500], [2000, 1700, 3999, 1501], 4, 2, 1),         # whole units
    ([2000, 1111, 300, 1500], [2000, 1700, 3999, 1501], 4, 2, 333),
    ([2500, 2000], [2003, 1999], 8, 1, 0),
]


@pytest.mark.parametrize("spread", [1.0, 40.0])
@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("case", SEVERAL, ids=lambda c: "x".join(map(str, c[0])) + f"_h{c[2]}x{c[3]}_b{c[4]}")
def test_several_long_sequences(ctx, case, cached, spread):
    """Each against its own reference: places of its rows, keys and ranges."""
    nq, nk, kv_heads, group, block = case
    q = normal(41, sum(nq), kv_heads * group, 128, spread=spread)
    k, v = normal(42, sum(nk), kv_heads, 128), normal(43, sum(nk), kv_heads, 128)
    got, k, v = attend(ctx, cached, q, k, v, nq, nk, block, max(nk) + 77)
    for s, x in enumerate(zip(parts(got, nq), parts(q, nq), parts(k, nk), parts(v, nk))):
        if nq[s]:
            R.assert_attention(x[0], *reference(*x[1:], block), f"sequence {s}")


@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("case", [
    ([1 + i * 7 % 5 for i in range(1000)], [1 + i * 11 % 90 for i in range(1000)], 1, 2, 64),
    ([i % 3 for i in range(700)], [i * 13 % 70 for i in range(700)], 2, 1, 128),
    ([1] * 3000, [1 + i * 17 % 40 for i in range(3000)], 1, 4, 64),
    ([400] + [1] * 63, [500] + [1 + 3 * i for i in range(63)], 1, 4, 128),      # a prompt beside single tokens
    ([1] * 20 + [500], [1 + 30 * i for i in range(20)] + [500], 1, 4, 128),
], ids=lambda c: f"{len(c[0])}x{max(c[0])}_d{c[4]}")
def test_many_sequences(ctx, case, cached):
    nq, nk, kv_heads, group, d = case
    q = normal(51, sum(nq), kv_heads * group, d)
    k, v = normal(52, sum(nk), kv_heads, d), normal(53, sum(nk), kv_heads, d)
    got, k, v = attend(ctx, cached, q, k, v, nq, nk, 1)
    q, k, v = q.cpu(), k.cpu(), v.cpu()
    refs = [R.attention(*x, 1) for x in zip(parts(q, nq), parts(k, nk), parts(v, nk))]
    R.assert_attention(got, *(torch.cat([r[i] for r in refs]) for i in range(2)), f"{len(nq)} sequences")


# --- scales of a cache's values -----------------------------------------------------------------------

@pytest.mark.parametrize("far", [125, 100])
@pytest.mark.parametrize("seqs,n,d,what", [(40, 16, 64, "few rows"), (40, 16, 128, "few rows"), (2, 320, 64, "32 rows"),
                                           (2, 320, 128, "32 rows"), (1, 1600, 128, "64 rows")])
def test_every_scale_beside_any_other(ctx, seqs, n, d, what, far):
    """A row that sees one key returns its value exactly, at every scale, whatever scales stand beside it: the
    kernels leave the codes of neighbouring tokens in bits that the conversion does not look at.  With 2^125 (as
    accumulators) the 64-row kernel takes its second pass, with 2^100 its first."""
    total = seqs * n
    g = torch.Generator(device="cuda")
    g.manual_seed(61)
    pick = lambda hi, *shape: torch.randint(0, hi, shape, generator=g, device="cuda")  # noqa: E731
    k = (2 * pick(2, total, 1, d) - 1).to(BF)              # signs: far apart from one another, and stored as they are
    steps = torch.tensor([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda", dtype=torch.float64)[pick(7, total, 1, d)]
    steps.unflatten(-1, (-1, 32))[..., 0] = 6.0            # (fixes the scale of the 32 dims)
    scale = torch.exp2(pick(2 * far + 1, total, 1, d // 32).double() - far).repeat_interleave(32, -1)
    v = (steps * scale * (2 * pick(2, total, 1, d) - 1)).to(BF)
    order = torch.cat([torch.randperm(n, generator=g, device="cuda") + s * n for s in range(seqs)])
    q = k[order] * 64.0                                     # logits 64 d for its key, and less by 300 and more (log2) else
    cache = ctx.qcache(seqs, 1, d, n)
    ctx.qcache_append(cache, k, v, ints([0] * seqs))
    got = ctx.qcache_attention(cache, q, ints([n] * seqs), causal_block=0)
    assert torch.equal(got, v[order])


# --- far places and any workspace ----------------------------------------------------------------------

FAR = (1 << 21) + (1 << 14) + 5        # tokens: 8 heads of 128 dims, or 16 of 64, pass 2^31 elements and 2^32 bytes


@pytest.mark.parametrize("what", ["queries", "keys"])
@pytest.mark.parametrize("nq,nk,d", [(300, 500, 64), (300, 500, 128), (200, 1700, 128)])
def test_packed_rows_behind_32_bit_offsets(ctx, nq, nk, d, what):
    """One sequence at the end of large tensors, whose other rows belong to none."""
    heads = 1024 // d
    at_q, at_k = (FAR, 0) if what == "queries" else (0, FAR)
    q = torch.empty(at_q + nq, heads, d, dtype=BF, device="cuda")
    k, v = (torch.empty(at_k + nk, heads, d, dtype=BF, device="cuda") for _ in range(2))
    q[at_q:], k[at_k:], v[at_k:] = normal(71, nq, heads, d), normal(72, nk, heads, d), normal(73, nk, heads, d)
    out = torch.empty_like(q)
    out[max(at_q - 8, 0):at_q] = 9.0
    ctx.packed_attention(q, k, v, ints([at_q, at_q + nq]), ints([at_k, at_k + nk]), out=out, causal_block=1)
    assert bool((out[max(at_q - 8, 0):at_q] == 9.0).all())
    R.assert_attention(out[at_q:], *reference(q[at_q:], k[at_k:], v[at_k:], 1))


@pytest.mark.parametrize("rows", [1, 100, 1400])
@pytest.mark.parametrize("d,capacity", [(64, 1 << 17), (128, 1 << 17), (128, 1000)])
def test_cached_attention_behind_32_bit_offsets(ctx, d, capacity, rows):
    """The last sequences of a cache of more than 2^32 bytes; the others are empty.  (1400 rows for each of 3 are
    more than 32 for each of the 68 or 128 that a long capacity makes: those run on the tile kernels.)"""
    seqs, heads = (1 << 32) // (2 * capacity * d * 17 // 32) // 4 + 8, 4
    cache = ctx.qcache(seqs, heads, d, capacity)
    assert cache.data.numel() > 1 << 32
    longest = min(capacity, 2000)
    nk = [0] * (seqs - 3) + [longest, longest // 3, longest - 1]
    nq = [0] * (seqs - 3) + [rows, rows, rows]
    k, v = normal(74, sum(nk), heads, d), normal(75, sum(nk), heads, d)
    start, cu = torch.zeros(seqs, dtype=torch.int32, device="cuda"), offsets(nk)
    ctx.qcache_append(cache, k, v, start, cu_seqlens=cu)
    ctx.qcache_read(cache, k, v, start, cu_seqlens=cu)
    q = normal(76, 3 * rows, 2 * heads, d)
    got = ctx.qcache_attention(cache, q, ints(nk), offsets(nq), causal_block=1)
    refs = [reference(*x, 1) for x in zip(parts(q, nq[-3:]), parts(k, nk[-3:]), parts(v, nk[-3:]))]
    R.assert_attention(got, *(torch.cat([r[i] for r in refs]) for i in range(2)))


def test_rotation_and_append_of_rows_behind_32_bit_offsets(ctx):
    heads, d, n = 8, 128, FAR
    x = torch.zeros(n, heads, d, dtype=BF, device="cuda")
    tail = normal(77, 100, heads, d)
    x[-100:] = tail
    cache = ctx.qcache(1, heads, d, 100)
    cu = ints([n - 100, n])
    ctx.qcache_append(cache, x, x, ints([0]), cu_seqlens=cu)
    k, v = torch.zeros_like(tail), torch.zeros_like(tail)
    ctx.qcache_read(cache, k, v, ints([0]))
    want = R.stored(tail.cpu())
    assert torch.equal(k.cpu().double(), want) and torch.equal(v.cpu().double(), want)
    ctx.rotate(x, x, axis_dims=(44, 42, 42), grid=(45, 80), frame0=2)
    pos = R.grid_positions(n, 45, 80, 2)[:, -100:]
    ref = R.rotate(tail.cpu(), pos, (44, 42, 42))
    assert float(tail.abs().max()) < 6
    # half a step of the output; sines 2.8e-7 and three roundings of 2^-24 of two products of inputs up to 6
    assert bool(((x[-100:].cpu().double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 12 * (2.8e-7 + 3 * 2.0 ** -24)).all())
    assert bool((x[:100] == 0).all())


@pytest.mark.parametrize("fill", [0, 255, 127])
@pytest.mark.parametrize("cached,nq,nk,d", [(True, [1, 0, 1], [4000, 900, 3], 128), (True, [90, 100, 1], [3000, 0, 2000], 64),
                                            (False, [90, 0, 100], [3000, 70, 2000], 128)])
def test_any_workspace(ctx, cached, nq, nk, d, fill):
    """What a workspace held before, NaN or large values, reaches no result."""
    q, k, v = normal(81, sum(nq), 4, d), normal(82, sum(nk), 2, d), normal(83, sum(nk), 2, d)
    want, _, _ = attend(ctx, cached, q, k, v, nq, nk, 1)
    work = torch.full((64 << 20,), fill, dtype=torch.uint8, device="cuda")
    if cached:
        cache = ctx.qcache(3, 2, d, max(nk))
        ctx.qcache_append(cache, k, v, ints([0] * 3), cu_seqlens=offsets(nk))
        got = ctx.qcache_attention(cache, q, ints(nk), offsets(nq), causal_block=1, workspace=work)
    else:
        got = ctx.packed_attention(q, k, v, offsets(nq), offsets(nk), causal_block=1, workspace=work)
    assert torch.equal(got, want) and bool((work != fill).any())


@pytest.mark.parametrize("d", [64, 128])
def test_equal_parts_of_queries_over_keys_by_offsets(ctx, d):
    nk = [30, 200, 0, 77]
    q, k, v = normal(84, 4 * 50, 4, d), normal(85, sum(nk), 2, d), normal(86, sum(nk), 2, d)
    got = ctx.packed_attention(q, k, v, None, offsets(nk), n_seqs=4)
    refs = [reference(*x, 0) for x in zip(parts(q, [50] * 4), parts(k, nk), parts(v, nk))]
    R.assert_attention(got, *(torch.cat([r[i] for r in refs]) for i in range(2)))
