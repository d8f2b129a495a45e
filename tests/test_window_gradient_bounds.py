"""The bounds of tests/gradient_bounds.py on the CPU: gradients computed with the roundings that they allow for pass, and zeroed,
negated, or 5% long or short ones do not."""
import pytest
import torch

import gradient_bounds as B
import window_ref as W

SHAPES = [(40, 40, 64, (1, 9, 3)), (200, 200, 64, (1, 0, 0)), (130, 300, 128, (1, 100, 7)), (150, 150, 128, (37, 74, 0)), (90, 90, 128, (0, 0, 0))]


def rounded(x):
    return x.to(torch.bfloat16).double()


def in_bf16(q, k, v, do, mask):
    """Gradients with p, ds, the output and the results in bf16."""
    s = q.shape[-1] ** -0.5
    q, k, v, do = (t[:, 0].double() for t in (q, k, v, do))
    p = torch.softmax((q @ k.T * s).masked_fill(~mask, -1e30), -1).masked_fill(~mask, 0.0)
    out = rounded(rounded(p) @ v / rounded(p).sum(1, keepdim=True).clamp(min=1e-30))
    ds = rounded(p * (do @ v.T - (do * out).sum(1, keepdim=True)))
    return [rounded(t).unsqueeze(1) for t in (ds @ k * s, ds.T @ q * s, rounded(p).T @ do)]


@pytest.mark.parametrize("n,m,dim,mask", SHAPES)
def test_bounds_tell_right_from_wrong(n, m, dim, mask):
    block, window, sinks = mask
    g = torch.Generator().manual_seed(5)
    q, k, v, do = (torch.randn(r, 1, dim, generator=g).to(torch.bfloat16) for r in (n, m, m, n))
    seen = W.sees(n, m, block, window, sinks)
    right = [t for t, _ in W.gradients(q, k, v, do, seen).values()]
    value = lambda *x: (W.attention(*x, seen)[0] * do.double()).sum()  # noqa: E731
    for i, (want, got) in enumerate(zip(right, in_bf16(q, k, v, do, seen))):
        at = [t.double() for t in (q, k, v)]
        by = lambda x, i=i, at=at: value(*at[:i], x, *at[i + 1:])  # noqa: E731
        print(f"{B.share(got, want):.5f}")
        assert B.share(got, want) < B.BOUND
        assert B.along(got, by, at[i])
        for wrong in (torch.zeros_like(got), -got, 1.05 * got, 0.95 * got, 2 * got):
            assert B.share(wrong, want) > B.BOUND
            assert not B.along(wrong, by, at[i])
