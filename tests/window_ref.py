"""Plain 64-bit forms of the operators of a model with a sliding window, for their tests, with how far a result
in fewer bits may be off: norm with rotary positions and its gradients, attention with a window and first
tokens and its gradients.  torch on the CPU, loops over sequences and heads; no code of the library."""
import math

import torch

import operators_ref as R

F64 = torch.float64
# cosines and sines: 8.5e-8 of the instruction, 2^-25 of a turn; two products and a sum in 32 bits
TURN = 8.5e-8 + 2 * math.pi * 2.0 ** -25 + 3 * 2.0 ** -24
# the norm: a sum of up to 256 squares over 16 products a lane and 5 exchanges, at most 22 roundings of 2^-24, of which the
# root keeps half; the root itself 2^-23, eps and the mean 2 more, and two products: under 2^-20 in all
NORM = 2.0 ** -20


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def pair_size(x, axis_dims, halves):
    """|a| + |b| of the pair that each dim turns with; 0 for dims that do not turn."""
    rot = sum(axis_dims)
    a = x.abs().to(F64)
    size = torch.zeros_like(a)
    if halves:
        size[..., :rot] = (a[..., :rot // 2] + a[..., rot // 2:rot]).repeat(1, 1, 2)
    else:
        size[..., :rot] = (a[..., 0:rot:2] + a[..., 1:rot:2]).repeat_interleave(2, -1)
    return size


def norm_rotate(x, w, pos, axis_dims, out_type, eps=1e-6, **kw):
    """(y, tolerance) of x [tokens][heads][d], w [d] or None."""
    x = x.to(F64)
    w = torch.ones(x.shape[-1], dtype=F64) if w is None else w.to(F64)
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    z = x * r * w
    y = R.rotate(z, pos, axis_dims, **kw)
    far = float(pos.abs().max())
    size = pair_size(z, axis_dims, kw.get("halves", False))
    tol = size * (TURN + far * 2.0 ** -51 + NORM) + y.abs() * (NORM + half_step(out_type)) + 1e-30
    return y, tol


def norm_rotate_backward(x, w, dout, pos, axis_dims, eps=1e-6, inverse=False, **kw):
    """(dx, tolerance, dw, tolerance)."""
    kind, d = x.dtype, x.shape[-1]
    x, dout = x.to(F64), dout.to(F64)
    w = torch.ones(d, dtype=F64) if w is None else w.to(F64)
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n = x * r
    g1 = R.rotate(dout, pos, axis_dims, inverse=not inverse, **kw)
    far = float(pos.abs().max())
    off = pair_size(dout, axis_dims, kw.get("halves", False)) * (TURN + far * 2.0 ** -51)      # of g1
    g = g1 * w
    mean = (g * n).mean(-1, keepdim=True)
    dx = r * (g - n * mean)
    # every factor of the products is off by NORM at most, and the sum over dims adds as many roundings as the norm's
    dmean = ((off * w.abs() + 2 * NORM * g.abs()) * n.abs()).mean(-1, keepdim=True)
    tol = r * (off * w.abs() + n.abs() * dmean + 2 * NORM * (g.abs() + n.abs() * mean.abs())) + dx.abs() * (NORM + half_step(kind)) + 1e-30
    # sums over tokens and heads: a thread's, a work group's slots, 32 threads': 256 additions at most at the tests' sizes
    dw = (g1 * n).sum((0, 1))
    tol_w = ((off + 2 * NORM * g1.abs()) * n.abs()).sum((0, 1)) + (g1 * n).abs().sum((0, 1)) * 2.0 ** -16 + 1e-30
    return dx, tol, dw, tol_w


def sees(n, m, block, window, sinks):
    """[n][m] truth values, query by query."""
    out = torch.zeros(n, m, dtype=torch.bool)
    for i in range(n):
        p = m - n + i
        if block == 0:
            out[i] = True
            continue
        if p < 0:
            continue
        e = (p // block + 1) * block
        out[i, :max(0, min(e, m))] = True
        if window and e - window > sinks:
            out[i, sinks:max(sinks, e - window)] = False
    return out


def attention(q, k, v, mask, scale=None):
    """One sequence: q [n][heads][d], k, v [m][kv heads][d], mask [n][m].  Returns (output, sum p |v|, lse, p)."""
    n, heads, d = q.shape
    m, kv_heads = k.shape[0], k.shape[1]
    out, mag = torch.zeros(n, heads, d, dtype=F64), torch.zeros(n, heads, d, dtype=F64)
    lse, probs = torch.full((heads, n), -math.inf, dtype=F64), torch.zeros(heads, n, m, dtype=F64)
    if n == 0 or m == 0:
        return out, mag, lse, probs
    blind = ~mask.any(1, keepdim=True)
    for h in range(heads):
        kh, vh = k[:, h // (heads // kv_heads)].to(F64), v[:, h // (heads // kv_heads)].to(F64)
        logits = (q[:, h].to(F64) @ kh.T * (scale if scale else d ** -0.5)).masked_fill(~mask, -math.inf)
        lse[h] = torch.logsumexp(logits, 1)
        p = torch.softmax(logits, -1).masked_fill(blind, 0.0)
        hide = ~mask                                # (values that nobody sees may be anything)
        shown = torch.where(hide.all(0).unsqueeze(1), 0.0, vh)
        out[:, h], mag[:, h], probs[h] = p @ shown, p @ shown.abs(), p
    return out, mag, lse, probs


def gradients(q, k, v, dout, mask, scale=None):
    """{name: (gradient, tolerance)} of one sequence.

    The tolerances.  The logarithms of the row sums are off by 2^-8 (sums of probabilities that are rounded to bf16, by
    2^-8 at most), so that p formed again is off by that factor, and by 2^-14 for logits in 32 bits; it is rounded once more
    for the products: 2^-7 (1.01) in all.  delta = rowsum(dout out) takes the output as rounded: it is off by at
    most sum |dout| (tolerance of the output).  ds = p (dp - delta) is off by p's factor, by p times what
    delta is off, and by dp's sum in 32 bits (2^-14 of the sum of magnitudes); it is rounded once more, 2^-8."""
    n, heads, d = q.shape
    m, kv_heads = k.shape[0], k.shape[1]
    group = heads // kv_heads
    s = scale if scale else d ** -0.5
    out, mag, _, probs = attention(q, k, v, mask, scale)
    far = R.attention_tolerance(out, mag)
    zeros = lambda t: torch.zeros(t.shape, dtype=F64)  # noqa: E731
    dq, dk, dv, tq, tk, tv = zeros(q), zeros(k), zeros(v), zeros(q), zeros(k), zeros(v)
    factor = 2.0 ** -7 * 1.02 + 2.0 ** -13
    for h in range(heads):
        qh, kh, vh, do = q[:, h].to(F64), k[:, h // group].to(F64), v[:, h // group].to(F64), dout[:, h].to(F64)
        p = probs[h]
        dp, delta = do @ vh.T, (do * out[:, h]).sum(1, keepdim=True)
        ds = p * (dp - delta)
        e = p * ((do.abs() * far[:, h]).sum(1, keepdim=True) + 2.0 ** -14 * (do.abs() @ vh.abs().T)) * 1.02 + factor * ds.abs()
        dq[:, h] = ds @ kh * s
        tq[:, h] = e @ kh.abs() * s
        dk[:, h // group] += ds.T @ qh * s
        tk[:, h // group] += e.T @ qh.abs() * s
        dv[:, h // group] += p.T @ do
        tv[:, h // group] += factor * (p.T @ do.abs())
    return {name: (g, t + 2.0 ** -8 * g.abs() + 1e-30) for name, g, t in (("dq", dq, tq), ("dk", dk, tk), ("dv", dv, tv))}


def assert_close(got, want, tol, what=""):
    got = got.cpu().to(F64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got - want).abs()
    if off.numel():
        print(f"{what}: max err {float(off.max()):.3e}, of its tolerance {float((off / tol).max()):.3f}", flush=True)
    assert bool((off <= tol).all()), f"{what}: {int((off > tol).sum())} values off, by up to {float((off - tol).max()):.3e} too much"


def assert_attention(got, out, mag, what=""):
    if out.numel():
        R.assert_attention(got, out, mag, what)
