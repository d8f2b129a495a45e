"""Gradients of attention with a window as a whole (tests/gradient_bounds.py): their size and direction against the plain 64-bit
form, and against differences of the formula."""
import pytest

import gradient_bounds as B
import window_ref as W
from test_gpu_operators import ctx, normal, offsets, spaced  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def run(ctx, q, k, v, do, cu_q=None, cu_k=None, **kw):  # noqa: F811
    q, k, v, do = (spaced(t) for t in (q, k, v, do))
    lse = torch.empty(q.shape[1], q.shape[0], device="cuda")
    out = ctx.window_attention(q, k, v, cu_q, cu_k, lse=lse, **kw)
    return ctx.window_attention_backward(q, k, v, out, lse, do, cu_q, cu_k, **kw)


SHAPES = [
    # kv heads, group, queries, keys (None: the queries')
    (1, 1, [40], None),
    (2, 3, [33, 200, 64], None),
    (1, 4, [130, 60], [300, 90]),            # kept context
    (2, 1, [700], None),
    (1, 2, [30], [2500]),                    # key units in pieces, merged
]


@pytest.mark.parametrize("mask", [(0, 0, 0), (1, 0, 0), (1, 9, 3), (1, 100, 7), (37, 74, 0)], ids=lambda m: "block%d_window%d_sinks%d" % m)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}_{s[2][0]}x{(s[3] or s[2])[0]}")
def test_errors_are_small_as_a_whole(ctx, shape, dim, mask):  # noqa: F811
    kv_heads, group, queries, keys = shape
    block, window, sinks = mask
    lengths, heads = keys or queries, kv_heads * group
    q, k, v, do = (normal(980 + i, sum(n), h, dim) for i, (n, h) in enumerate(
        ((queries, heads), (lengths, kv_heads), (lengths, kv_heads), (queries, heads))))
    got = run(ctx, q, k, v, do, offsets(queries), offsets(lengths) if keys else None, causal_block=block, window=window, sinks=sinks)
    a = b = 0
    for n, m in zip(queries, lengths):
        want = W.gradients(q[a:a + n], k[b:b + m], v[b:b + m], do[a:a + n], W.sees(n, m, block, window, sinks))
        for t, (name, (g, _)) in zip(got, want.items()):
            lo, hi = (a, a + n) if name == "dq" else (b, b + m)
            off = B.share(t[lo:hi], g)
            print(f"{name} of {n} x {m}: {off:.5f}", flush=True)
            assert off <= B.BOUND, name
        a, b = a + n, b + m


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("mask", [(0, 0, 0), (1, 9, 3), (16, 48, 20)], ids=lambda m: "block%d_window%d_sinks%d" % m)
def test_gradients_are_as_long_as_differences_say(ctx, dim, mask):  # noqa: F811
    block, window, sinks = mask
    n = 90
    q, k, v, do = (normal(990 + i, n, 1, dim) for i in range(4))
    seen = W.sees(n, n, block, window, sinks)
    at = [t.double() for t in (q, k, v)]
    for i, g in enumerate(run(ctx, q, k, v, do, causal_block=block, window=window, sinks=sinks)):
        assert B.along(g, lambda x: (W.attention(*at[:i], x, *at[i + 1:], seen)[0] * do.double()).sum(), at[i]), i
