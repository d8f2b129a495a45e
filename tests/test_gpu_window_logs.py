"""The logarithms of the row sums that attention with a window gives: of the probabilities in 32 bits, in every kernel
that writes them, and the probabilities that the gradients form again from them."""
import math

import pytest

import window_ref as W
from test_gpu_operators import ctx, normal, offsets  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

CASES = [
    # dim, kv heads, group, queries, keys (None: the queries'), spread of q and k
    (64, 2, 3, [5, 200, 0, 64, 1], None, 1.0),       # waves of 32 rows
    (128, 2, 2, [257, 1, 129], None, 1.0),
    (64, 1, 2, [100, 3], [0, 250], 1.0),             # rows that see nothing
    (128, 1, 4, [130, 40], [300, 7], 6.0),
    (128, 2, 1, [1700], None, 1.0),                  # waves of 64 rows
    (128, 2, 1, [1700], None, 8.0),                  # the same with a running maximum
    (128, 24, 1, [1400], None, 1.0),                 # 264 units
    (64, 2, 2, [40], [3000], 1.0),                   # ranges of keys, merged: few of them, and many
    (128, 2, 2, [40], [3000], 1.0),
    (64, 2, 2, [5], [20000], 1.0),
    (128, 2, 2, [5], [20000], 8.0),
]


@pytest.mark.parametrize("mask", [(0, 0, 0), (1, 0, 0), (1, 700, 3), (16, 33, 40)], ids=lambda m: "block%d_window%d_sinks%d" % m)
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}_{c[1]}x{c[2]}_{c[3][0]}x{(c[4] or c[3])[0]}_{c[5]:g}")
def test_logarithms_are_of_sums_in_32_bits(ctx, case, mask):  # noqa: F811
    """How far they may be off, with a the scale times the sum of a logit's products' magnitudes:
    * a logit's products are exact and added up in 32 bits, 16 at a time: up to 2^-24 a for each of 8 instructions, and as
      much inside them: 2^-20 a;
    * the scale times log2 e is rounded three times, a logit less the maximum and the maximum once: 2^-22 of the largest
      logit; an exponential by 2^-23, the logarithm and its product with ln 2 by 2^-23 of themselves and 2^-23;
    * a row's sum of m numbers, half of them in a lane of its own: 2^-24 (m / 2 + 8) of it, and 2^-24 for each of up to 32
      ranges."""
    dim, kv_heads, group, queries, keys, spread = case
    block, window, sinks = mask
    lengths, heads = keys or queries, kv_heads * group
    q, k = (normal(900 + i, sum(n), h, dim, spread=spread) for i, (n, h) in enumerate(((queries, heads), (lengths, kv_heads))))
    v = normal(902, sum(lengths), kv_heads, dim)
    lse = torch.full((heads, sum(queries)), math.nan, device="cuda")
    ctx.window_attention(q.cuda(), k.cuda(), v.cuda(), offsets(queries), offsets(lengths) if keys else None, lse=lse,
                         causal_block=block, window=window, sinks=sinks)
    lse = lse.cpu().double()
    a = b = 0
    for n, m in zip(queries, lengths):
        blind = ~W.sees(n, m, block, window, sinks)
        for h in sorted({0, heads // 2, heads - 1}):
            got = lse[h, a:a + n]
            if m == 0 or n == 0:
                assert bool((got == -math.inf).all())
                continue
            qs, ks = q[a:a + n, h].double(), k[b:b + m, h // group].double()
            logits = (qs @ ks.T * dim ** -0.5).masked_fill(blind, -math.inf)
            size = (qs.abs() @ ks.abs().T * dim ** -0.5).masked_fill(blind, 0.0).amax(1)
            want = torch.logsumexp(logits, 1)
            assert torch.equal(got == -math.inf, blind.all(1))
            seen = ~blind.all(1)
            tol = size * (2.0 ** -20 + 2.0 ** -22) + want.abs() * 2.0 ** -22 + 2.0 ** -22 + (m / 2 + 40) * 2.0 ** -24
            off = (got - want).abs()[seen]
            if off.numel():
                print(f"{n} x {m} head {h}: max err {float(off.max()):.2e}, of its tolerance {float((off / tol[seen]).max()):.3f}", flush=True)
            assert bool((off <= tol[seen]).all()), (float(off.max()), float((off / tol[seen]).max()))
        a, b = a + n, b + m


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [90, 1700])
def test_a_row_that_sees_one_key_weighs_it_by_one(ctx, dim, tokens):  # noqa: F811
    """The first token of a causal sequence sees itself.  Formed again from its logarithm its probability is off by 2^-20 of its
    logit's magnitudes (see above), far less than the 2^-9 that bf16 rounds to 1: with an output gradient in the first
    row alone, dv of that token is that row, bit for bit, and of the others zero."""
    q, k, v, do = (normal(920 + i, 2 * tokens, 6, dim) for i in range(4))
    do[1:tokens] = 0
    do[tokens + 1:] = 0
    q, k, v, do = (t.cuda() for t in (q, k, v, do))
    cu = offsets([tokens, tokens])
    lse = torch.empty(6, 2 * tokens, device="cuda")
    out = ctx.window_attention(q, k, v, cu, lse=lse)
    assert torch.equal(out[0], v[0]) and torch.equal(out[tokens], v[tokens])
    _, _, dv = ctx.window_attention_backward(q, k, v, out, lse, do, cu)
    assert torch.equal(dv, do)
