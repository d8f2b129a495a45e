"""Plain 64-bit forms of the operators beside the routed attention, for their tests: rotary
positions, the 4-bit cache's values, attention with per-query key counts.  torch on the CPU,
loops over sequences and heads; no code of the library."""
import math

import torch

F64 = torch.float64
CODES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)


def rotate(x, pos, axis_dims, theta=10000.0, halves=False, joint=False, inverse=False):
    """x [tokens][heads][d], pos [axes][tokens]."""
    y = x.to(F64).clone()
    rot = sum(axis_dims)
    pair = 0
    for axis, m in enumerate(axis_dims):
        for j in range(m // 2):
            share = 2.0 * pair / rot if joint else 2.0 * j / m
            angle = pos[axis].to(F64) * theta ** -share * (-1.0 if inverse else 1.0)
            c, s = angle.cos().unsqueeze(1), angle.sin().unsqueeze(1)
            u, w = (pair, pair + rot // 2) if halves else (2 * pair, 2 * pair + 1)
            a, b = x[..., u].to(F64), x[..., w].to(F64)
            y[..., u], y[..., w] = a * c - b * s, a * s + b * c
            pair += 1
    return y


def grid_positions(n, grid_h, grid_w, frame0):
    t = torch.arange(n)
    return torch.stack([frame0 + t // (grid_h * grid_w), t // grid_w % grid_h, t % grid_w])


def stored(x):
    """The values a 4-bit cache holds for x [..., d]: by search over all values of each group's scale."""
    g = x.to(F64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    out = torch.empty_like(g)
    flat, res = g.reshape(-1, 32), out.reshape(-1, 32)
    for i in range(flat.shape[0]):
        row = flat[i]
        if not torch.isfinite(row).all():
            res[i] = math.nan
            continue
        top = float(row.abs().max())
        if top == 0.0:
            res[i] = 0.0
            continue
        k = math.frexp(top)[1] - 1                       # 2^k <= top < 2^(k + 1)
        e = min(max(k - 2 if top <= 1.75 * 2.0 ** k else k - 1, -125), 125)
        far = (row.abs().unsqueeze(1) - CODES * 2.0 ** e).abs()
        best = far.min(1).values
        # on a tie the even code
        pick = torch.stack([(far[:, c] == best) * (2 if c % 2 == 0 else 1) for c in range(8)], 1).argmax(1)
        res[i] = CODES[pick] * 2.0 ** e * torch.sign(row)
    return out.reshape(x.shape)


def seen(n, m, block):
    """Keys that each of n queries sees of m."""
    if block == 0:
        return [m] * n
    return [0 if m - n + i < 0 else min(m, ((m - n + i) // block + 1) * block) for i in range(n)]


def attention(q, k, v, block=0, scale=None):
    """One sequence: q [n][heads][d], k, v [m][kv heads][d].  Returns (output, sum p |v|)."""
    n, heads, d = q.shape
    m, kv_heads = k.shape[0], k.shape[1]
    out, mag = torch.zeros(n, heads, d, dtype=F64), torch.zeros(n, heads, d, dtype=F64)
    if n == 0 or m == 0:
        return out, mag
    count = torch.tensor(seen(n, m, block)).unsqueeze(1)
    hidden = torch.arange(m) >= count
    for h in range(heads):
        kh, vh = k[:, h // (heads // kv_heads)].to(F64), v[:, h // (heads // kv_heads)].to(F64)
        logits = q[:, h].to(F64) @ kh.T * (scale if scale else d ** -0.5)
        p = torch.softmax(logits.masked_fill(hidden, -math.inf), -1)
        p = torch.where(count == 0, torch.zeros_like(p), p)
        out[:, h], mag[:, h] = p @ vh, p @ vh.abs()
    return out, mag


def attention_tolerance(out, mag):
    """How far an attention output in bf16 may be off: half a step of the result (2^-8 of it), and
    the rounding of the probabilities to bf16.  The latter are rounded by factors within 1 +- 2^-8
    in the numerator and in the row sum alike, which moves the quotient by at most
    2 * 2^-8 / (1 - 2^-8) of sum p |v|; logits and sums in 32 bits add less than 2^-14 of it."""
    return 2.0 ** -8 * out.abs() + (2.0 ** -7 * 1.01 + 2.0 ** -14) * mag + 1e-30


def assert_attention(got, out, mag, what=""):
    got = got.cpu().to(F64)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - out).abs() - attention_tolerance(out, mag)
    print(f"{what}: max err {float((got - out).abs().max()):.3e}", flush=True)
    assert bool((over <= 0).all()), f"{what}: {int((over > 0).sum())} values off, by up to {float(over.max()):.3e} too much"
