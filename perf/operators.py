"""Operators around the routed attention, as cases to be timed.

* ``rotate``  rotary positions over several axes (time, height, width) of a block's queries and
              keys: `Context.rotate`;
* ``append``  storing new keys and values in a cache of 4-bit values and reading them back:
              `Context.qcache_append`, `Context.qcache_read`;
* ``cached``  attention of new queries over such a cache: `Context.qcache_attention`;
* ``packed``  attention over whole prompts or clips packed behind one another, with grouped heads
              and a causal or block-causal mask: `Context.packed_attention`.

The 4-bit values: 32 neighbouring dims of one token share a power of two, and each is one of
0, 1/2, 1, 3/2, 2, 3, 4, 6 times it, with a sign.  Query i of n over m keys sits at position
p = m - n + i; with `block` = 0 it sees every key, else the keys before (p // block + 1) * block,
so that 1 is the causal mask and a block of tokens sees itself and all earlier blocks.
"""
import math

import torch

own = False

GROUP = 32                       # dims that share a scale
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LOW, HIGH = -125, 125            # range of the scale's exponent


# --- cases -------------------------------------------------------------------------------------

def _rotate(name, tokens, heads, kv_heads, dim, **more):
    c = dict(op="rotate", name=name, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, gh=0, gw=0, far=0,
             halves=False, joint=False, inverse=False, theta=10000.0, x="bf16", out="bf16", head_major=True)
    c.update(more)
    return c


def _append(name, seqs, tokens, heads, dim, capacity, **more):
    return dict(dict(op="append", name=name, seqs=seqs, tokens=tokens, heads=heads, dim=dim, capacity=capacity,
                     ragged=False), **more)


def _cached(name, seqs, queries, kv_heads, group, dim, capacity, **more):
    return dict(dict(op="cached", name=name, seqs=seqs, queries=queries, kv_heads=kv_heads, group=group, dim=dim,
                     capacity=capacity, ragged=False, block=1), **more)


def _packed(name, seqs, tokens, kv_heads, group, dim, **more):
    return dict(dict(op="packed", name=name, seqs=seqs, tokens=tokens, keys=0, kv_heads=kv_heads, group=group,
                     dim=dim, ragged=False, block=1), **more)


def listed():
    return [
        # the smallest block of the tests: two frames of 8x8 tokens, where launches are all there is
        _rotate("rotate_tiny", 128, 4, 4, 64, gh=8, gw=8),
        # queries and keys of a 720P block as a projection writes them (token by token), rotated
        # into the head-major layout that the routed attention reads
        _rotate("rotate_block_720p", 10800, 12, 12, 128, gh=45, gw=80),
        # the gradient's direction in 32 bits: far positions given one by one, pairs half a head apart
        _rotate("rotate_back_far", 4099, 16, 4, 128, far=1 << 20, halves=True, joint=True, inverse=True,
                theta=1e6, x="f32", out="f32", head_major=False),
        # one new token for each of 64 sequences
        _append("append_step", 64, 64, 8, 128, 4096),
        # the block of a denoising step at 720P, into its place in a seven-block window
        _append("append_block_720p", 1, 10800, 12, 128, 75600),
        # one token of one sequence over a long cache
        _cached("decode_long", 1, 1, 8, 4, 128, 131072),
        # one token for each sequence of a batch, lengths from 1 to 8192, a group of odd size
        _cached("decode_ragged", 48, 48, 4, 7, 64, 8192, ragged=True),
        # a 480P block over its full window
        _cached("window_480p", 1, 4680, 12, 1, 128, 32760, block=0),
        # a short prompt, as a text encoder's decoder half reads it
        _packed("prompt_short", 1, 77, 12, 1, 64),
        # prompts of different lengths behind one another, four query heads to a key head
        _packed("prompts_ragged", 9, 16000, 8, 4, 128, ragged=True),
        # a clip of four 480P blocks: a block sees itself and the blocks before it
        _packed("clip_480p", 1, 18720, 12, 1, 128, block=4680),
        # two 480P blocks, each over its own text of up to 512 tokens
        _packed("blocks_over_text", 2, 9360, 12, 1, 128, keys=739, ragged=True, block=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("rotate", "append", "cached", "cached", "packed", "packed"))
        dim = rng.choice((64, 128, 128))
        if op == "rotate":
            c = _rotate("", _log_int(rng, 1, 12000), rng.choice((1, 4, 12, 16, 24)), rng.choice((0, 1, 4, 12)), dim,
                        halves=rng.random() < 0.5, joint=rng.random() < 0.3, inverse=rng.random() < 0.4,
                        theta=rng.choice((1e4, 1e6)), x=rng.choice(("bf16", "bf16", "f32")),
                        out=rng.choice(("bf16", "bf16", "f32")), head_major=rng.random() < 0.5)
            if rng.random() < 0.5:
                c["gh"], c["gw"] = rng.randint(3, 68), rng.randint(3, 120)
            else:
                c["far"] = _log_int(rng, 64, 1 << 20)
        elif op == "append":
            seqs = _log_int(rng, 1, 64)
            each = _log_int(rng, 1, 12000)
            c = _append("", seqs, seqs * each, rng.choice((1, 2, 4, 8, 12)), dim, each + _log_int(rng, 1, 4000),
                        ragged=rng.random() < 0.5)
            if c["tokens"] * c["heads"] > 12 * 10800:
                continue
        elif op == "cached":
            if rng.random() < 0.6:      # single tokens
                seqs = _log_int(rng, 1, 64)
                c = _cached("", seqs, seqs, rng.choice((1, 2, 4, 8, 12)), rng.choice((1, 3, 4, 7, 8)), dim,
                            _log_int(rng, 1, 131072), ragged=rng.random() < 0.6, block=rng.choice((0, 1)))
                if c["seqs"] * c["kv_heads"] * c["capacity"] > 8 * 131072:
                    continue
            else:
                seqs = _log_int(rng, 1, 6)
                each = _log_int(rng, 2, 4800)
                c = _cached("", seqs, seqs * each, rng.choice((1, 2, 4, 12)), rng.choice((1, 2, 3, 4)), dim,
                            each + _log_int(rng, 1, 24000), ragged=rng.random() < 0.6,
                            block=rng.choice((0, 1, 1, each // 3 + 1)))
        else:
            seqs = _log_int(rng, 1, 24)
            each = _log_int(rng, 2, 6000)
            c = _packed("", seqs, seqs * each, rng.choice((1, 2, 4, 8, 12)), rng.choice((1, 1, 2, 3, 4)), dim,
                        ragged=rng.random() < 0.7, block=rng.choice((0, 1, 1, 1, each // 4 + 1)))
            if rng.random() < 0.25:
                c["keys"] = seqs * _log_int(rng, 1, 600)
            if c["tokens"] > 40000:
                continue
        if work(c)["flops"] > work(listed()[7])["flops"] or _plain_bytes(c) > 20e9:
            continue
        del c["name"]
        return c


def _split(total, parts, seed):
    """`parts` lengths that add up to `total`, from very short to very long ones."""
    g = torch.Generator()
    g.manual_seed(seed)
    share = torch.exp(3.0 * torch.rand(parts, generator=g, dtype=torch.float64))
    cut = torch.floor(torch.cumsum(share, 0) / share.sum() * total).to(torch.int64)
    cut[-1] = total
    return torch.diff(cut, prepend=torch.zeros(1, dtype=torch.int64))


def _lengths(case):
    """(queries, keys) of every sequence, on the host: a property of the case, not of the seed."""
    n = case["seqs"]
    even = lambda total: torch.full((n,), total // n, dtype=torch.int64)  # noqa: E731
    if case["op"] == "append":
        return (_split(case["tokens"], n, 1).clamp(max=case["capacity"]) if case["ragged"] else even(case["tokens"])), None
    if case["op"] == "cached":
        queries = even(case["queries"])
        if not case["ragged"]:
            return queries, torch.full((n,), case["capacity"], dtype=torch.int64)
        g = torch.Generator()
        g.manual_seed(2)
        return queries, (torch.rand(n, generator=g, dtype=torch.float64) * case["capacity"]).to(torch.int64) + 1
    queries = _split(case["tokens"], n, 3) if case["ragged"] else even(case["tokens"])
    if not case["keys"]:
        return queries, queries
    return queries, _split(case["keys"], n, 4) if case["ragged"] else even(case["keys"])


def _plain_bytes(case):
    """Memory of the plain form's logits."""
    if case["op"] not in ("cached", "packed"):
        return 0
    nq, nk = _lengths(case)
    return 4.0 * case["seqs"] * case["kv_heads"] * case["group"] * int(nq.max()) * int(nk.max())


def work(case):
    d = case["dim"]
    if case["op"] == "rotate":
        size = {"bf16": 2, "f32": 4}
        values = case["tokens"] * (case["heads"] + case["kv_heads"]) * d
        given = case["tokens"] * 12 if case["far"] else 0
        return {"bytes": values * (size[case["x"]] + size[case["out"]]) + given, "flops": 3 * values}
    stored = d // 2 + d // GROUP
    if case["op"] == "append":
        n, _ = _lengths(case)
        rows = int(n.sum()) * case["heads"] * 2
        return {"bytes": rows * 2 * (2 * d + stored), "flops": rows * d * 4}
    nq, nk = _lengths(case)
    heads = case["kv_heads"] * case["group"]
    pairs = 0
    for n, m in zip(nq.tolist(), nk.tolist()):
        if case["block"] == 0:
            pairs += n * m
        else:
            p = torch.arange(m - n, m, dtype=torch.int64).clamp(min=-1)
            seen = torch.where(p < 0, 0, (p // case["block"] + 1) * case["block"]).clamp(max=m)
            pairs += int(seen.sum())
    moved = int(nq.sum()) * heads * d * 2 * 2
    each = 2 * d if case["op"] == "packed" else stored
    return {"bytes": moved + int(nk.sum()) * case["kv_heads"] * 2 * each, "flops": 4 * d * heads * pairs}


# --- inputs ------------------------------------------------------------------------------------

def _axis_dims(d):
    """How a head's dims are shared by time, height and width: what is left of thirds goes to time."""
    return [d - 4 * (d // 6), 2 * (d // 6), 2 * (d // 6)]


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _offsets(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(n, 0)]).to(torch.int32).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    bf16 = torch.bfloat16
    d = case["dim"]
    s = {"case": case}
    if own:
        from paper_2607_20125_amd import headcast
        s["ctx"] = headcast.Context(headcast.default_config())
    if case["op"] == "rotate":
        kinds = {"bf16": bf16, "f32": torch.float32}
        n = case["tokens"]
        heads = [h for h in (case["heads"], case["kv_heads"]) if h]
        s["x"] = [_normal(gen, (n, h, d), kinds[case["x"]]) for h in heads]
        # [tokens][heads][dims] of an output that is laid out as the case says
        s["out"] = [torch.empty((h, n, d) if case["head_major"] else (n, h, d), dtype=kinds[case["out"]], device="cuda")
                    for h in heads]
        s["view"] = [o.transpose(0, 1) if case["head_major"] else o for o in s["out"]]
        s["frame0"] = int(torch.randint(0, 100, (1,), generator=gen, device="cuda"))
        s["positions"] = torch.randint(0, case["far"], (3, n), generator=gen, device="cuda", dtype=torch.int32) if case["far"] else None
        return s
    nq, nk = _lengths(case)
    if case["op"] == "append":
        heads, total = case["heads"], int(nq.sum())
        s["cu"] = _offsets(nq) if case["ragged"] else None
        room = (case["capacity"] - nq).to(torch.float64)
        at = torch.rand(len(nq), generator=gen, device="cuda", dtype=torch.float64).cpu()
        s["start"] = torch.floor(at * (room + 1)).to(torch.int32).cuda()
        seq = torch.repeat_interleave(torch.arange(len(nq)), nq)
        place = torch.arange(total) - (torch.cumsum(nq, 0) - nq)[seq]
        s["seq"], s["slot"] = seq.cuda(), place.cuda() + s["start"].long()[seq.cuda()]
        s["k"], s["v"] = _normal(gen, (total, heads, d), bf16), _normal(gen, (total, heads, d), bf16)
        if own:
            s["cache"] = s["ctx"].qcache(case["seqs"], heads, d, case["capacity"])
            s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        else:
            s["codes"] = torch.zeros((2, case["seqs"], case["capacity"], heads, d // 2), dtype=torch.uint8, device="cuda")
            s["scales"] = torch.zeros((2, case["seqs"], case["capacity"], heads, d // GROUP), dtype=torch.int8, device="cuda")
        return s
    kv_heads, heads = case["kv_heads"], case["kv_heads"] * case["group"]
    s["nq"], s["nk"] = nq.cuda(), nk.cuda()
    s["most_q"], s["most_k"] = int(nq.max()), int(nk.max())
    s["cu_q"] = _offsets(nq)
    s["q"] = _normal(gen, (int(nq.sum()), heads, d), bf16)
    s["out"] = torch.empty_like(s["q"])
    if case["op"] == "packed":
        s["cu_k"] = _offsets(nk)
        s["k"], s["v"] = (_normal(gen, (int(nk.sum()), kv_heads, d), bf16) for _ in range(2))
        return s
    seqs, cap = case["seqs"], case["capacity"]
    k, v = (_normal(gen, (seqs * cap, kv_heads, d), bf16) for _ in range(2))
    s["kv_len"] = nk.to(torch.int32).cuda()
    if own:
        s["cache"] = s["ctx"].qcache(seqs, kv_heads, d, cap)
        s["ctx"].qcache_append(s["cache"], k, v, torch.zeros(seqs, dtype=torch.int32, device="cuda"))
    else:
        s["stored"] = [_store(x.view(seqs, cap, kv_heads, d)) for x in (k, v)]
    return s


# --- plain forms -------------------------------------------------------------------------------

def _store(x):
    """(two codes a byte, exponents of the scales) of x [..., d]."""
    g = x.float().unflatten(-1, (-1, GROUP))
    mantissa, exponent = torch.frexp(g.abs().amax(-1, keepdim=True))      # mantissa in [1/2, 1)
    # 7/4 of a power of two still rounds to 6 with half a step's error, so it needs no larger scale
    e = torch.where(2 * mantissa <= 1.75, exponent - 3, exponent - 2).clamp(LOW, HIGH)
    y = torch.ldexp(g, -e)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = torch.where(y < 0, code + 8, code).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), e.squeeze(-1).to(torch.int8)


def _values(codes, scales):
    """The values that codes and scales stand for."""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float32, device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    return torch.ldexp(table[c.int()].unflatten(-1, (-1, GROUP)), scales.int().unsqueeze(-1)).flatten(-2)


def _angles(case, s):
    """Angles [tokens][1][pairs] in 64 bits."""
    n, dims = case["tokens"], _axis_dims(case["dim"])
    if case["far"]:
        pos = s["positions"].double()
    else:
        t = torch.arange(n, device="cuda")
        frame = case["gh"] * case["gw"]
        pos = torch.stack([s["frame0"] + t // frame, t % frame // case["gw"], t % case["gw"]]).double()
    freq = []
    for a, m in enumerate(dims):
        at = torch.arange(m // 2, device="cuda", dtype=torch.float64) + (sum(dims[:a]) // 2 if case["joint"] else 0)
        freq.append(case["theta"] ** (-2.0 * at / (sum(dims) if case["joint"] else m)))
    return torch.cat([pos[a].unsqueeze(-1) * f for a, f in enumerate(freq)], -1).unsqueeze(1)


def _turn(x, cos, sin, halves):
    if halves:
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _padded(x, starts, lengths, most):
    """[seqs][most][heads][d] of a packed tensor; what is behind a sequence's end is zero."""
    i = torch.arange(most, device=x.device)
    at = (starts.long().unsqueeze(1) + i).clamp(max=max(x.shape[0] - 1, 0))
    return torch.where((i < lengths.unsqueeze(1))[..., None, None], x[at].float(), 0.0)


def _attend(q, k, v, nq, nk, block, group):
    """q [seqs][n][heads][d] over k, v [seqs][m][kv heads][d], in 32 bits."""
    seqs, n, heads, d = q.shape
    m = k.shape[1]
    i, j = torch.arange(n, device=q.device), torch.arange(m, device=q.device)
    p = (nk - nq).unsqueeze(1) + i
    seen = nk.unsqueeze(1).expand(seqs, n)
    if block:
        seen = torch.where(p < 0, 0, torch.minimum(seen, (p // block + 1) * block))
    q = q.unflatten(2, (heads // group, group)).permute(0, 2, 3, 1, 4).reshape(seqs, heads // group, group * n, d)
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.transpose(1, 2).contiguous()
    logits = torch.matmul(q * (1.0 / math.sqrt(d)), k).view(seqs, heads // group, group, n, m)
    hidden = (j >= seen.unsqueeze(-1))[:, None, None]
    logits.masked_fill_(hidden, -math.inf)
    top = logits.amax(-1, keepdim=True)
    logits.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = logits.sum(-1, keepdim=True)
    o = torch.matmul(logits.flatten(2, 3), v).view(seqs, heads // group, group, n, d)
    return (o / torch.where(total == 0, 1.0, total)).permute(0, 3, 1, 2, 4).reshape(seqs, n, heads, d)


def _unpadded(o, lengths):
    return o[torch.arange(o.shape[1], device=o.device) < lengths.unsqueeze(1)].to(torch.bfloat16)


def run(s):
    case = s["case"]
    if case["op"] == "rotate":
        if own:
            s["ctx"].rotate(s["x"], s["view"], axis_dims=_axis_dims(case["dim"]), positions=s["positions"],
                            grid=None if case["far"] else (case["gh"], case["gw"]), frame0=s["frame0"], theta=case["theta"],
                            halves=case["halves"], joint=case["joint"], inverse=case["inverse"])
            return s["out"]
        angle = _angles(case, s)
        cos, sin = angle.cos().float(), (-angle if case["inverse"] else angle).sin().float()
        for x, view in zip(s["x"], s["view"]):
            view.copy_(_turn(x.float(), cos, sin, case["halves"]))
        return s["out"]
    if case["op"] == "append":
        if own:
            s["ctx"].qcache_append(s["cache"], s["k"], s["v"], s["start"], cu_seqlens=s["cu"])
            s["ctx"].qcache_read(s["cache"], s["k_out"], s["v_out"], s["start"], cu_seqlens=s["cu"])
            return s["k_out"], s["v_out"]
        codes, scales = _store(torch.stack([s["k"], s["v"]]))
        s["codes"][:, s["seq"], s["slot"]] = codes
        s["scales"][:, s["seq"], s["slot"]] = scales
        back = _values(s["codes"][:, s["seq"], s["slot"]], s["scales"][:, s["seq"], s["slot"]]).to(torch.bfloat16)
        return back[0], back[1]
    if case["op"] == "cached":
        if own:
            return s["ctx"].qcache_attention(s["cache"], s["q"], s["kv_len"], cu_seqlens=s["cu_q"], out=s["out"],
                                             causal_block=case["block"])
        k, v = (_values(*x) for x in s["stored"])
        live = (torch.arange(case["capacity"], device="cuda") < s["nk"].unsqueeze(1))[..., None, None]
        k, v = (torch.where(live, x, 0.0) for x in (k, v))
    else:
        if own:
            return s["ctx"].packed_attention(s["q"], s["k"], s["v"], s["cu_q"], cu_k=s["cu_k"] if case["keys"] else None,
                                             out=s["out"], causal_block=case["block"])
        k, v = (_padded(x, s["cu_k"][:-1], s["nk"], s["most_k"]) for x in (s["k"], s["v"]))
    q = _padded(s["q"], s["cu_q"][:-1], s["nq"], s["most_q"])
    return _unpadded(_attend(q, k, v, s["nq"], s["nk"], case["block"], case["group"]), s["nq"])


# --- the definition in 64 bits -------------------------------------------------------------------

def _nearest(x):
    """The stored value nearest to each of x, with an even code on ties."""
    g = x.double().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    power = torch.floor(torch.log2(top.clamp(min=1e-300)))
    power = power - (torch.exp2(power) > top).double() + (torch.exp2(power + 1) <= top).double()
    scale = torch.exp2((power - 2 + (top > 1.75 * torch.exp2(power)).double()).clamp(LOW, HIGH))
    best, off = torch.zeros_like(g), g.abs()
    for code in (2, 4, 6, 1, 3, 5, 7):     # even codes first: a later one has to be nearer
        far = (g.abs() - VALUES[code] * scale).abs()
        best, off = torch.where(far < off, VALUES[code] * scale, best), torch.minimum(far, off)
    return (best * torch.sign(g)).flatten(-2)


def _meaning(codes, scales):
    """What codes and scales stand for: a sign, two bits of exponent and one of mantissa, the smallest exponent without its leading one."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).to(torch.int64)
    exponent, half = (c // 2) % 4, (c % 2).double() / 2
    size = torch.where(exponent == 0, half, (1 + half) * torch.exp2(exponent.double() - 1))
    shared = torch.repeat_interleave(torch.exp2(scales.double()), GROUP, dim=-1)
    return torch.where(c >= 8, -size, size) * shared


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "rotate":
        n, d, dims = case["tokens"], case["dim"], _axis_dims(case["dim"])
        if case["far"]:
            pos = s["positions"].double().T
        else:
            t = torch.arange(n, device="cuda")
            y = t // case["gw"]
            pos = torch.stack([s["frame0"] + y // case["gh"], y % case["gh"], t - y * case["gw"]], -1).double()
        turn = torch.empty(n, 1, d // 2, dtype=torch.complex128, device="cuda")
        first = 0
        for axis, m in enumerate(dims):
            for pair in range(m // 2):
                share = 2 * (first + pair) / d if case["joint"] else 2 * pair / m
                angle = pos[:, axis] * math.exp(-share * math.log(case["theta"]))
                turn[:, 0, first + pair] = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)
            first += m // 2
        found = []
        for x in s["x"]:
            x = x.double()
            pairs = torch.stack(x.chunk(2, -1), -1) if case["halves"] else x.unflatten(-1, (-1, 2))
            y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            y = torch.cat([y[..., 0], y[..., 1]], -1) if case["halves"] else y.flatten(-2)
            found.append(y.transpose(0, 1).contiguous() if case["head_major"] else y)
        return found
    if case["op"] == "append":
        return _nearest(s["k"]), _nearest(s["v"])
    if work(case)["flops"] > 2e12:
        return None
    nq, nk = (x.tolist() for x in _lengths(case))
    cu_q, group, d = s["cu_q"].tolist(), case["group"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        n, m = nq[b], nk[b]
        if case["op"] == "cached":
            k, v = (_meaning(*(part[b, :m] for part in x)) for x in s["stored"])
        else:
            first = sum(nk[:b])
            k, v = (s[x][first:first + m].double() for x in ("k", "v"))
        q = s["q"][cu_q[b]:cu_q[b] + n].double()
        at = m - n + torch.arange(n, device="cuda")
        seen = torch.full_like(at, m) if case["block"] == 0 else ((at // case["block"] + 1) * case["block"]).clamp(0, m)
        seen = torch.where(at < 0, 0, seen) if case["block"] else seen
        mask = torch.arange(m, device="cuda") < seen.unsqueeze(1)
        for h in range(case["kv_heads"] * group):
            logits = (q[:, h] @ k[:, h // group].T) / math.sqrt(d)
            p = torch.softmax(logits.masked_fill(~mask, -math.inf), -1)
            out[cu_q[b]:cu_q[b] + n, h] = torch.where(mask.any(-1, keepdim=True), p, 0.0) @ v[:, h // group]
    return out
