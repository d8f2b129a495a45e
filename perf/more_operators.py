"""Operators of a model with a sliding window, as cases to be timed: before, in and behind the attention.

* ``norm``       root-mean-square norm of every head of a block's queries and keys, then rotary
                 positions, in one pass: `Context.norm_rotate`;
* ``norm_back``  its gradients, of the inputs and of the weights: `Context.norm_rotate_backward`;
* ``store``      new keys and values into the pages of a cache: `Context.paged_append`;
* ``paged``      attention of a chunk of new tokens, or of single ones, over such a cache, with a
                 window and first tokens that stay visible: `Context.paged_attention`;
* ``window``     the same over whole prompts or clips packed behind one another: `Context.window_attention`;
* ``train``      that with the gradients of queries, keys and values: `Context.window_attention`, then
                 `Context.window_attention_backward`.

The mask: query i of n over m keys sits at position p = m - n + i, and with `block` = c > 0 its
keys end before e = (p // c + 1) * c (none if p < 0).  Of these it sees the first `sinks`, and
those from e - `window` on (all of them if `window` is 0).  c = 1 is the causal mask; with c a block's
tokens and a window of whole blocks, a block sees itself, the blocks before it that the window holds, and
the first block or tokens of the sequence.  `block` = 0 is no mask.
"""
import math

import torch

own = False

EPS = 1e-6


# --- cases -------------------------------------------------------------------------------------

def _norm(name, tokens, heads, kv_heads, dim, **more):
    c = dict(op="norm", name=name, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, gh=0, gw=0, far=0,
             halves=False, joint=False, theta=10000.0, x="bf16", out="bf16", weight="bf16", head_major=True)
    c.update(more)
    return c


def _store(name, seqs, tokens, heads, dim, capacity, page, **more):
    return dict(dict(op="store", name=name, seqs=seqs, tokens=tokens, heads=heads, dim=dim, capacity=capacity,
                     page=page, ragged=False), **more)


def _paged(name, seqs, queries, kv_heads, group, dim, capacity, page, **more):
    return dict(dict(op="paged", name=name, seqs=seqs, tokens=queries, kv_heads=kv_heads, group=group, dim=dim,
                     capacity=capacity, page=page, ragged=False, block=1, window=0, sinks=0), **more)


def _window(name, op, seqs, tokens, kv_heads, group, dim, **more):
    return dict(dict(op=op, name=name, seqs=seqs, tokens=tokens, keys=0, kv_heads=kv_heads, group=group,
                     dim=dim, ragged=False, block=1, window=0, sinks=0), **more)


def listed():
    return [
        # the smallest block of the tests: two frames of 8x8 tokens, where launches are all there is
        _norm("norm_tiny", 128, 4, 4, 64, gh=8, gw=8),
        # queries and keys of a 720P block as a projection writes them, into the head-major layout
        # that the routed attention reads
        _norm("norm_block_720p", 10800, 12, 12, 128, gh=45, gw=80),
        # the gradient of a 480P block's, from the attention's layout back to the projection's
        _norm("norm_back_block_480p", 4680, 12, 12, 128, op="norm_back", gh=30, gw=52),
        # in 32 bits: far positions given one by one, pairs half a head apart, grouped heads
        _norm("norm_back_far", 4099, 16, 4, 128, op="norm_back", far=1 << 20, halves=True, joint=True, theta=1e6,
              x="f32", out="f32", weight="f32", head_major=False),
        # one new token for each of 64 sequences, pages of 16 tokens
        _store("store_step", 64, 64, 8, 128, 512, 16),
        # the block of a denoising step at 480P, into its place in a seven-block window
        _store("store_block_480p", 1, 4680, 12, 128, 32760, 64),
        # one token of one sequence over all of a long cache
        _paged("step_long", 1, 1, 8, 4, 128, 131072, 64),
        # one token for each sequence of a batch, lengths from 1 to 8192, a group of odd size; the window
        # has passed most pages, which are gone
        _paged("step_ragged", 48, 48, 4, 7, 64, 8192, 16, ragged=True, window=2048, sinks=64),
        # chunks of prompts of different lengths, each over what its window and first tokens leave of the cache
        _paged("chunk_ragged", 5, 2500, 8, 4, 128, 16384, 32, ragged=True, window=4096, sinks=128),
        # a clip of four 480P blocks: a block sees itself, the one before it and the first
        _window("clip_480p", "window", 1, 18720, 12, 1, 128, block=4680, window=9360, sinks=4680),
        # a batch of short texts of different lengths, three query heads to a key head, a few first tokens
        _window("train_prompts", "train", 6, 4000, 4, 3, 64, ragged=True, window=512, sinks=4),
        # training on a clip of three 480P blocks: a block sees itself and the first
        _window("train_clip_480p", "train", 1, 14040, 12, 1, 128, block=4680, window=4680, sinks=4680),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mask(rng, longest):
    """A mask for sequences of up to about `longest` keys."""
    block = rng.choice((1, 1, 1, longest // 4 + 1))
    kind = rng.choice(("all", "window", "window", "sinks", "sinks"))
    return dict(block=block if kind != "all" else rng.choice((0, 1)),
                window=0 if kind == "all" else _log_int(rng, 1, longest) if block == 1 else block * rng.randint(1, 3),
                sinks=0 if kind != "sinks" else _log_int(rng, 1, 200) if block == 1 else block)


def draw(rng):
    while True:
        op = rng.choice(("norm", "norm_back", "store", "paged", "paged", "window", "train", "train"))
        dim = rng.choice((64, 128, 128))
        if op in ("norm", "norm_back"):
            x = rng.choice(("bf16", "bf16", "f32"))
            c = _norm("", _log_int(rng, 1, 12000), rng.choice((1, 4, 12, 16, 24)), rng.choice((0, 1, 4, 12)), dim, op=op,
                      halves=rng.random() < 0.5, joint=rng.random() < 0.3, theta=rng.choice((1e4, 1e6)), x=x,
                      out=rng.choice(("bf16", "bf16", "f32")), weight=rng.choice((x, "f32")), head_major=rng.random() < 0.5)
            if rng.random() < 0.5:
                c["gh"], c["gw"] = rng.randint(3, 68), rng.randint(3, 120)
            else:
                c["far"] = _log_int(rng, 64, 1 << 20)
        elif op == "store":
            seqs, each = _log_int(rng, 1, 64), _log_int(rng, 1, 8000)
            c = _store("", seqs, seqs * each, rng.choice((1, 2, 4, 8, 12)), dim, each + _log_int(rng, 1, 4000),
                       rng.choice((16, 32, 64, 128, 256)), ragged=rng.random() < 0.5)
            if c["tokens"] * c["heads"] > 12 * 10800 or seqs * c["capacity"] * c["heads"] > 400000:
                continue
        elif op == "paged":
            if rng.random() < 0.6:      # single tokens
                seqs = _log_int(rng, 1, 64)
                c = _paged("", seqs, seqs, rng.choice((1, 2, 4, 8, 12)), rng.choice((1, 3, 4, 7, 8)), dim,
                           _log_int(rng, 1, 131072), rng.choice((16, 32, 64, 128)), ragged=rng.random() < 0.6)
                if seqs * c["kv_heads"] * c["capacity"] > 8 * 131072:
                    continue
            else:
                seqs, each = _log_int(rng, 1, 6), _log_int(rng, 2, 4800)
                c = _paged("", seqs, seqs * each, rng.choice((1, 2, 4, 12)), rng.choice((1, 2, 3, 4)), dim,
                           each + _log_int(rng, 1, 24000), rng.choice((16, 32, 64, 256)), ragged=rng.random() < 0.6)
            c.update(_mask(rng, c["capacity"]))
        else:
            seqs, each = _log_int(rng, 1, 24), _log_int(rng, 2, 6000)
            c = _window("", op, seqs, seqs * each, rng.choice((1, 2, 4, 8, 12)), rng.choice((1, 1, 2, 3, 4)), dim,
                        ragged=rng.random() < 0.7)
            c.update(_mask(rng, each))
            if rng.random() < 0.25:      # context that is kept from before, or fewer keys than queries
                c["keys"] = seqs * _log_int(rng, 1, 2 * each)
            if c["tokens"] > 40000:
                continue
        if work(c)["flops"] > work(listed()[-1])["flops"] or _plain_bytes(c) > 20e9:
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
    if case["op"] == "store":
        return (_split(case["tokens"], n, 1).clamp(max=case["capacity"]) if case["ragged"] else even(case["tokens"])), None
    if case["op"] == "paged":
        queries = even(case["tokens"])
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
    if case["op"] not in ("paged", "window", "train"):
        return 0
    nq, nk = _lengths(case)
    return (2.0 if case["op"] == "train" else 1.0) * 4 * case["seqs"] * case["kv_heads"] * case["group"] * int(nq.max()) * int(nk.max())


def _ends(case, n, m):
    """(ends, sinks, starts) of n queries over m keys: query i sees keys before sinks[i] and from starts[i] to ends[i]."""
    p = torch.arange(m - n, m, dtype=torch.int64)
    if case["block"] == 0:
        ends, starts = torch.full_like(p, m), torch.zeros_like(p)
    else:
        e = (torch.div(p, case["block"], rounding_mode="floor") + 1) * case["block"]
        ends = torch.where(p < 0, 0, e.clamp(max=m))
        starts = (e - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(p)
        starts = torch.minimum(starts, ends)
    return ends, torch.minimum(starts, torch.full_like(starts, case["sinks"])), starts


def work(case):
    d = case["dim"]
    size = {"bf16": 2, "f32": 4}
    if case["op"] in ("norm", "norm_back"):
        values = case["tokens"] * (case["heads"] + case["kv_heads"]) * d
        given = case["tokens"] * 12 if case["far"] else 0
        if case["op"] == "norm":
            return {"bytes": values * (size[case["x"]] + size[case["out"]]) + given, "flops": 7 * values}
        return {"bytes": values * (2 * size[case["x"]] + size[case["out"]]) + given, "flops": 14 * values}
    nq, nk = _lengths(case)
    if case["op"] == "store":
        rows = int(nq.sum()) * case["heads"] * 2
        return {"bytes": rows * 2 * 2 * d, "flops": rows * d}
    heads = case["kv_heads"] * case["group"]
    pairs, keys = 0, 0
    for n, m in zip(nq.tolist(), nk.tolist()):
        ends, sinks, starts = _ends(case, n, m)
        pairs += int((ends - starts + sinks).sum())
        if n:      # keys that any query sees
            keys += int(torch.cat([ends, sinks]).max() - max(0, int(starts.min()) - int(sinks.max()))) if int(ends.max()) else 0
    q, kv = int(nq.sum()) * heads * d * 2, keys * case["kv_heads"] * d * 2
    if case["op"] == "train":
        return {"bytes": 4 * q + 4 * kv, "flops": 14 * d * heads * pairs}
    return {"bytes": 2 * q + 2 * kv, "flops": 4 * d * heads * pairs}


# --- inputs ------------------------------------------------------------------------------------

KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def _axis_dims(d):
    """How a head's dims are shared by time, height and width: what is left of thirds goes to time."""
    return [d - 4 * (d // 6), 2 * (d // 6), 2 * (d // 6)]


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _offsets(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(n, 0)]).to(torch.int32).cuda()


def _tables(gen, seqs, pages):
    """Which page holds which run of a sequence's tokens: all in an order of their own, a few pages unused."""
    total = seqs * pages
    order = torch.randperm(total + 3, generator=gen, device="cuda")[:total]
    return order.to(torch.int32).view(seqs, pages), total + 3


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    bf16 = torch.bfloat16
    d = case["dim"]
    s = {"case": case}
    if own:
        from paper_2607_20125_amd import headcast
        s["ctx"] = headcast.Context(headcast.default_config())
    if case["op"] in ("norm", "norm_back"):
        n = case["tokens"]
        heads = [h for h in (case["heads"], case["kv_heads"]) if h]
        # projections before a norm: heads of different sizes
        s["x"] = [(3.0 * torch.rand((1, h, 1), generator=gen, device="cuda") + 0.2).mul(_normal(gen, (n, h, d), torch.float32)).to(KINDS[case["x"]])
                  for h in heads]
        s["weight"] = [(1.0 + 0.3 * _normal(gen, (d,), torch.float32)).to(KINDS[case["weight"]]) for _ in heads]
        s["frame0"] = int(torch.randint(0, 100, (1,), generator=gen, device="cuda"))
        s["positions"] = torch.randint(0, case["far"], (3, n), generator=gen, device="cuda", dtype=torch.int32) if case["far"] else None
        shape = lambda h: (h, n, d) if case["head_major"] else (n, h, d)  # noqa: E731
        if case["op"] == "norm":
            s["out"] = [torch.empty(shape(h), dtype=KINDS[case["out"]], device="cuda") for h in heads]
        else:
            s["out"] = [_normal(gen, shape(h), KINDS[case["out"]]) for h in heads]      # gradients of the outputs
            s["dx"] = [torch.empty_like(x) for x in s["x"]]
        # [tokens][heads][dims] of a tensor that is laid out as the case says
        s["view"] = [o.transpose(0, 1) if case["head_major"] else o for o in s["out"]]
        return s
    nq, nk = _lengths(case)
    if case["op"] in ("store", "paged"):
        page = case["page"]
        per = -(-case["capacity"] // page)
        s["table"], n_pages = _tables(gen, case["seqs"], per)
        kv_heads = case["heads"] if case["op"] == "store" else case["kv_heads"]
        shape = (n_pages, kv_heads, page, d)
        s["kp"], s["vp"] = (torch.zeros(shape, dtype=bf16, device="cuda") if case["op"] == "store" else _normal(gen, shape, bf16)
                            for _ in range(2))
        if own:
            s["pages"] = headcast.Pages(s["kp"].transpose(1, 2), s["vp"].transpose(1, 2))
    if case["op"] == "store":
        total = int(nq.sum())
        s["cu"] = _offsets(nq) if case["ragged"] else None
        room = (case["capacity"] - nq).to(torch.float64)
        at = torch.rand(len(nq), generator=gen, device="cuda", dtype=torch.float64).cpu()
        s["start"] = torch.floor(at * (room + 1)).to(torch.int32).cuda()
        seq = torch.repeat_interleave(torch.arange(len(nq)), nq)
        place = torch.arange(total) - (torch.cumsum(nq, 0) - nq)[seq]
        s["seq"], s["place"] = seq.cuda(), place.cuda()
        s["k"], s["v"] = _normal(gen, (total, case["heads"], d), bf16), _normal(gen, (total, case["heads"], d), bf16)
        return s
    kv_heads, heads = case["kv_heads"], case["kv_heads"] * case["group"]
    s["nq"], s["nk"] = nq.cuda(), nk.cuda()
    s["most_q"], s["most_k"] = int(nq.max()), int(nk.max())
    s["cu_q"], s["cu_k"] = _offsets(nq), _offsets(nk)
    s["q"] = _normal(gen, (int(nq.sum()), heads, d), bf16)
    s["out"] = torch.empty_like(s["q"])
    if case["op"] == "paged":
        s["kv_len"] = nk.to(torch.int32).cuda()
        # pages behind the end, and those that the window of the first new token has passed, are gone
        first = torch.arange(per, device="cuda").unsqueeze(0) * page
        p = s["nk"] - s["nq"]
        low = torch.clamp((p // max(case["block"], 1) + 1) * max(case["block"], 1) - case["window"], min=0) if case["window"] else torch.zeros_like(p)
        gone = (first >= s["nk"].unsqueeze(1)) | ((first >= case["sinks"]) & (first + page <= low.unsqueeze(1)))
        s["table"][gone] = -1
        return s
    s["k"], s["v"] = (_normal(gen, (int(nk.sum()), kv_heads, d), bf16) for _ in range(2))
    if case["op"] == "train":
        s["dout"] = _normal(gen, tuple(s["q"].shape), bf16)
        s["lse"] = torch.empty((heads, s["q"].shape[0]), dtype=torch.float32, device="cuda")
        s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
    return s


# --- plain forms -------------------------------------------------------------------------------

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


def _unpadded(o, lengths):
    return o[torch.arange(o.shape[1], device=o.device) < lengths.unsqueeze(1)].to(torch.bfloat16)


def _paged_rows(pages, table, most):
    """[seqs][most][heads][d] of the cache; a page that is gone gives any other's."""
    slot = torch.arange(most, device=pages.device)
    page = table.long().clamp(min=0)[:, slot // pages.shape[2]]
    return pages[page, :, slot % pages.shape[2]].float()


def _hidden(case, nq, nk, n, m):
    """[seqs][n][m]: keys that a query does not see."""
    i, j = torch.arange(n, device=nq.device), torch.arange(m, device=nq.device)
    p = (nk - nq).unsqueeze(1) + i
    if case["block"] == 0:
        return (j >= nk.view(-1, 1, 1)).expand(-1, n, -1)
    e = (p // case["block"] + 1) * case["block"]
    end = torch.where(p < 0, 0, torch.minimum(e, nk.unsqueeze(1))).unsqueeze(-1)
    hidden = j >= end
    if case["window"]:
        hidden = hidden | ((j >= case["sinks"]) & (j < (e - case["window"]).unsqueeze(-1)))
    return hidden


def _rows(x, group):
    """[seqs][kv heads][group * n][d] of [seqs][n][heads][d]."""
    x = x.unflatten(2, (x.shape[2] // group, group)).permute(0, 2, 3, 1, 4)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[4])


def _back(x, n):
    """[seqs][n][heads][d] of [seqs][kv heads][group * n][d]."""
    return x.unflatten(2, (-1, n)).permute(0, 3, 1, 2, 4).flatten(2, 3)


def _weights(case, s, q, k):
    """exp(logits - the row's largest) and the rows' sums, in 32 bits."""
    n, m = s["most_q"], s["most_k"]
    logits = torch.matmul(q * (1.0 / math.sqrt(case["dim"])), k.transpose(2, 3).contiguous())
    hidden = _hidden(case, s["nq"], s["nk"], n, m)
    logits.view(*logits.shape[:2], case["group"], n, m).masked_fill_(hidden[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    logits.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = logits.sum(-1, keepdim=True)
    return logits, torch.where(total == 0, 1.0, total)


def run(s):
    case = s["case"]
    if case["op"] in ("norm", "norm_back"):
        if own:
            at = dict(axis_dims=_axis_dims(case["dim"]), eps=EPS, positions=s["positions"],
                      grid=None if case["far"] else (case["gh"], case["gw"]), frame0=s["frame0"], theta=case["theta"],
                      halves=case["halves"], joint=case["joint"])
            if case["op"] == "norm":
                s["ctx"].norm_rotate(s["x"], s["weight"], s["view"], **at)
                return s["out"]
            dx, dweight = s["ctx"].norm_rotate_backward(s["x"], s["weight"], s["view"], s["dx"], **at)
            return {"dx": dx, "dweight": dweight}
        angle = _angles(case, s)
        cos, sin = angle.cos().float(), angle.sin().float()
        if case["op"] == "norm":
            for x, w, view in zip(s["x"], s["weight"], s["view"]):
                x = x.float()
                r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
                view.copy_(_turn(x * r * w.float(), cos, sin, case["halves"]))
            return s["out"]
        found = {"dx": [], "dweight": []}
        for x, w, view in zip(s["x"], s["weight"], s["view"]):
            kind, x = x.dtype, x.float()
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            x = x * r
            g = _turn(view.float(), cos, -sin, case["halves"])
            found["dweight"].append((g * x).double().sum((0, 1)).float())
            g = g * w.float()
            found["dx"].append((r * (g - x * (g * x).mean(-1, keepdim=True))).to(kind))
        return found
    if case["op"] == "store":
        if own:
            s["ctx"].paged_append(s["pages"], s["table"], s["k"], s["v"], s["start"], cu_seqlens=s["cu"])
        else:
            slot = s["start"].long()[s["seq"]] + s["place"]
            page = s["table"].long()[s["seq"], slot // case["page"]]
            s["kp"][page, :, slot % case["page"]] = s["k"]
            s["vp"][page, :, slot % case["page"]] = s["v"]
        return s["kp"], s["vp"]
    mask = dict(causal_block=case["block"], window=case["window"], sinks=case["sinks"])
    if own:
        if case["op"] == "paged":
            return s["ctx"].paged_attention(s["pages"], s["table"], s["q"], s["kv_len"], cu_seqlens=s["cu_q"], out=s["out"], **mask)
        cu_k = s["cu_k"] if case["keys"] else None
        if case["op"] == "window":
            return s["ctx"].window_attention(s["q"], s["k"], s["v"], s["cu_q"], cu_k, s["out"], **mask)
        s["ctx"].window_attention(s["q"], s["k"], s["v"], s["cu_q"], cu_k, s["out"], lse=s["lse"], **mask)
        dq, dk, dv = s["ctx"].window_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["cu_q"], cu_k,
                                                        s["dq"], s["dk"], s["dv"], **mask)
        return {"out": s["out"], "dq": dq, "dk": dk, "dv": dv}
    q = _rows(_padded(s["q"], s["cu_q"][:-1], s["nq"], s["most_q"]), case["group"])
    if case["op"] == "paged":
        k, v = (_paged_rows(x, s["table"], s["most_k"]) for x in (s["kp"], s["vp"]))
    else:
        k, v = (_padded(x, s["cu_k"][:-1], s["nk"], s["most_k"]) for x in (s["k"], s["v"]))
    k, v = (x.transpose(1, 2).contiguous() for x in (k, v))
    p, total = _weights(case, s, q, k)
    out = torch.matmul(p, v) / total
    whole = _unpadded(_back(out, s["most_q"]), s["nq"])
    if case["op"] != "train":
        return whole
    p.div_(total)
    do = _rows(_padded(s["dout"], s["cu_q"][:-1], s["nq"], s["most_q"]), case["group"])
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds.sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(case["dim"]))
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3), q)
    return {"out": whole, "dq": _unpadded(_back(dq, s["most_q"]), s["nq"]),
            "dk": _unpadded(dk.transpose(1, 2), s["nk"]), "dv": _unpadded(dv.transpose(1, 2), s["nk"])}


# --- the definition in 64 bits -------------------------------------------------------------------

def _exact_norm(case, s):
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
            turn[:, 0, first + pair] = torch.polar(torch.ones_like(angle), angle)
        first += m // 2

    def forward(x, w):
        y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS) * w
        pairs = torch.stack(y.chunk(2, -1), -1) if case["halves"] else y.unflatten(-1, (-1, 2))
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        return torch.cat([y[..., 0], y[..., 1]], -1) if case["halves"] else y.flatten(-2)

    found = {"dx": [], "dweight": []}
    outs = []
    for x, w, view in zip(s["x"], s["weight"], s["view"]):
        x, w = x.double().requires_grad_(), w.double().requires_grad_()
        y = forward(x, w)
        if case["op"] == "norm":
            y = y.detach()
            outs.append(y.transpose(0, 1).contiguous() if case["head_major"] else y)
        else:
            dx, dw = torch.autograd.grad(y, (x, w), view.double())
            found["dx"].append(dx)
            found["dweight"].append(dw)
    return outs if case["op"] == "norm" else found


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] in ("norm", "norm_back"):
        return _exact_norm(case, s)
    nq, nk = (x.tolist() if x is not None else None for x in _lengths(case))
    if case["op"] == "store":
        kp, vp = s["kp"].double(), s["vp"].double()
        table, start, at = s["table"].tolist(), s["start"].tolist(), 0
        for b, n in enumerate(nq):
            for first in range(n):
                if first and (start[b] + first) % case["page"]:
                    continue                     # stored with the rows before it
                slot = start[b] + first
                row, many = slot % case["page"], min(n - first, case["page"] - slot % case["page"])
                for pages, x in ((kp, s["k"]), (vp, s["v"])):
                    pages[table[b][slot // case["page"]], :, row:row + many] = x[at + first:at + first + many].double().transpose(0, 1)
            at += n
        return kp, vp
    if work(case)["flops"] > 4e12:
        return None
    cu_q, cu_k, group, d = s["cu_q"].tolist(), s["cu_k"].tolist(), case["group"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    if case["op"] == "train":
        dq = torch.zeros_like(out)
        dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(case["seqs"]):
        n, m = nq[b], nk[b]
        if n == 0 or m == 0:
            continue
        if case["op"] == "paged":
            k, v = (torch.cat([x[max(i, 0)] for i in s["table"][b].tolist()], 1)[:, :m].transpose(0, 1) for x in (s["kp"], s["vp"]))
        else:
            k, v = (s[x][cu_k[b]:cu_k[b + 1]] for x in ("k", "v"))
        q = s["q"][cu_q[b]:cu_q[b + 1]]
        at = torch.arange(m - n, m, device="cuda").unsqueeze(1)
        key = torch.arange(m, device="cuda").unsqueeze(0)
        sees = torch.ones(n, m, dtype=torch.bool, device="cuda")
        if case["block"]:
            # in units of blocks: a key's block is not behind the query's, and the window reaches back to it
            mine = torch.floor(at.double() / case["block"])
            sees = (at >= 0) & (torch.floor(key.double() / case["block"]) <= mine)
            if case["window"]:
                sees = sees & ((key < case["sinks"]) | (key >= (mine + 1) * case["block"] - case["window"]))
        blind = ~sees.any(1, keepdim=True)
        for h in range(case["kv_heads"] * group):
            qh, kh, vh = (x[:, i].double().requires_grad_(case["op"] == "train") for x, i in ((q, h), (k, h // group), (v, h // group)))
            p = torch.softmax((qh @ kh.T / math.sqrt(d)).masked_fill(~(sees | blind), -math.inf), -1).masked_fill(blind, 0.0)
            o = p @ vh
            out[cu_q[b]:cu_q[b + 1], h] = o.detach()
            if case["op"] == "train":
                gq, gk, gv = torch.autograd.grad(o, (qh, kh, vh), s["dout"][cu_q[b]:cu_q[b + 1], h].double())
                dq[cu_q[b]:cu_q[b + 1], h] = gq
                dk[cu_k[b]:cu_k[b + 1], h // group] += gk
                dv[cu_k[b]:cu_k[b + 1], h // group] += gv
    return {"out": out, "dq": dq, "dk": dk, "dv": dv} if case["op"] == "train" else out
