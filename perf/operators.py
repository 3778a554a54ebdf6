"""What the performance of the KV-cache operators is measured on: the calls that a serving step makes around the scheduler.

Three operators, in the order in which a step uses them:

  append   rotary positions on the new tokens' queries and keys, keys and values into the paged cache
  decode   attention of one new token per sequence over the paged cache, with the weight that every cached token got
  evict    a sequence's cache shortened to the tokens with the largest accumulated weight, copied to new pages

A cache is two tensors [pages, tokens of a page, heads, dim] (layout "hnd": the heads before the tokens in memory).
Lengths go by the case alone, values, page orders and positions by the seed.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
KEY_SCALE, VALUE_SCALE = 0.0625, 0.03125      # what one unit of an 8-bit cache stands for


def listed():
    return [
        # one sequence makes one token: latency
        dict(name="append_1", kind="append", tokens=1, q_heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, scaling="none",
             page=16, layout="nhd", x="bf16", cache="bf16", far=4096),
        # a decoding batch, half of each head rotated in neighbouring pairs, a long context's scaling, an 8-bit cache
        dict(name="append_193_e4m3", kind="append", tokens=193, q_heads=32, kv_heads=4, dim=128, rot=64, interleaved=True, scaling="yarn",
             page=32, layout="hnd", x="f16", cache="e4m3", far=131_072),
        # the uncached tokens of a batch of prompts, each cached token in a slot of its own
        dict(name="append_32768", kind="append", tokens=32_768, q_heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, scaling="ntk",
             page=1, layout="nhd", x="bf16", cache="bf16", far=16_384),
        # one short sequence: latency
        dict(name="decode_1_short", kind="decode", seqs=1, length=200, ragged=False, q_heads=32, kv_heads=8, dim=128, page=16, layout="nhd",
             x="bf16", cache="bf16", window=0, weight=False, shared=0),
        # an ordinary batch of odd lengths with an empty row, weights kept for eviction
        dict(name="decode_33_weight", kind="decode", seqs=33, length=8191, ragged=True, q_heads=32, kv_heads=8, dim=128, page=16,
             layout="nhd", x="bf16", cache="bf16", window=0, weight=True, shared=0),
        # slots of single tokens, as a radix tree hands them out; eight prompts of a group share their first 2,048 tokens
        dict(name="decode_64_radix", kind="decode", seqs=64, length=4096, ragged=True, q_heads=16, kv_heads=2, dim=64, page=1, layout="nhd",
             x="f16", cache="f16", window=0, weight=False, shared=2048),
        # two very long sequences in 8 bits: the work is split over the length
        dict(name="decode_2_long_e4m3", kind="decode", seqs=2, length=131_072, ragged=False, q_heads=32, kv_heads=4, dim=128, page=64,
             layout="hnd", x="bf16", cache="e4m3", window=0, weight=False, shared=0),
        # the largest: a full batch on long contexts, gigabytes of cache
        dict(name="decode_128_large", kind="decode", seqs=128, length=16_384, ragged=True, q_heads=32, kv_heads=8, dim=128, page=16,
             layout="nhd", x="bf16", cache="bf16", window=0, weight=False, shared=0),
        # a sliding window, every head with keys of its own, wide heads of an odd size
        dict(name="decode_16_window", kind="decode", seqs=16, length=5000, ragged=True, q_heads=8, kv_heads=8, dim=80, page=8, layout="hnd",
             x="bf16", cache="bf16", window=1024, weight=True, shared=0),
        # one short sequence is cut to a quarter
        dict(name="evict_1", kind="evict", seqs=1, length=1000, ragged=False, keep=250, sinks=4, recent=64, kv_heads=8, dim=128, page=16,
             layout="nhd", cache="bf16"),
        # a batch of odd lengths is cut to half of the longest; some rows are short enough to be kept whole
        dict(name="evict_32", kind="evict", seqs=32, length=8191, ragged=True, keep=4096, sinks=4, recent=512, kv_heads=8, dim=128, page=16,
             layout="nhd", cache="bf16"),
        # few and very long rows
        dict(name="evict_2_long_e4m3", kind="evict", seqs=2, length=131_072, ragged=False, keep=16_384, sinks=16, recent=2048, kv_heads=4,
             dim=128, page=64, layout="hnd", cache="e4m3"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "evict"])
    heads, dim, cache = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 128, 128, 192, 256]), rng.choice(["bf16", "f16", "e4m3"])
    c = dict(kind=kind, kv_heads=heads, dim=dim, page=rng.choice([1, 8, 16, 64]), layout=rng.choice(["nhd", "hnd"]), cache=cache)
    if kind != "evict":
        c["q_heads"] = heads * rng.choice([1, 2, 4, 5, 8, 16])
        c["x"] = cache if cache != "e4m3" else rng.choice(["bf16", "f16"])
    if kind == "append":
        c.update(tokens=_log(rng, 1, 12_000), rot=rng.choice([dim, dim, dim // 2, 16]), interleaved=rng.random() < 0.5,
                 scaling=rng.choice(["none", "linear", "ntk", "yarn"]), far=_log(rng, 128, 1 << 20))
        return c
    total = _log(rng, 64, 400_000)                       # cached tokens of the batch
    seqs = _log(rng, 1, max(1, min(128, total // 16)))
    length = max(1, min(131_072, total // seqs))
    c.update(seqs=seqs, length=length, ragged=rng.random() < 0.7)
    if kind == "decode":
        c.update(window=_log(rng, 16, length) if length > 64 and rng.random() < 0.25 else 0, weight=rng.random() < 0.5,
                 shared=length // 2 if rng.random() < 0.3 else 0)
    else:
        keep = max(1, min(length, int(length * rng.uniform(0.1, 0.9))))
        sinks = min(keep, rng.choice([0, 1, 4, 16]))
        c.update(keep=keep, sinks=sinks, recent=min(keep - sinks, int(keep * rng.uniform(0.0, 0.5))))
    return c


def lengths_of(case):
    """A ragged batch has lengths spread over [1, length] and, from eight sequences on, one row without any token."""
    n, top = case["seqs"], case["length"]
    if not case["ragged"]:
        return [top] * n
    got = [1 + int(((i + 1) * 0.6180339887498949) % 1.0 * top) for i in range(n)]
    got = [min(x, top) for x in got]
    got[0] = top
    if n >= 8:
        got[n // 2] = 0
    return got


def shared_pages(case):
    return case.get("shared", 0) // case["page"]


def _pages(case):
    """For every sequence the numbers of its pages, before they are shuffled: a group of eight shares its first pages."""
    page, lead, rows, used, heads = case["page"], shared_pages(case), [], 0, {}
    for i, n in enumerate(lengths_of(case)):
        need = -(-n // page)
        row = []
        if lead:
            if i // 8 not in heads:
                heads[i // 8] = list(range(used, used + lead))
                used += lead
            row = heads[i // 8][:min(lead, need)]
        fresh = need - len(row)
        rows.append(row + list(range(used, used + fresh)))
        used += fresh
    return rows, used


def _cache(g, pages, case, dev):
    t = TYPES[case["cache"]]
    shape = [pages, case["page"], case["kv_heads"], case["dim"]]
    mem = shape if case["layout"] == "nhd" else [shape[0], shape[2], shape[1], shape[3]]
    got = []
    for scale in (KEY_SCALE, VALUE_SCALE):
        x = torch.empty(mem, dtype=torch.bfloat16 if t == torch.bfloat16 else torch.float16, device=dev).normal_(generator=g)
        if case["cache"] == "e4m3":
            x = torch.cat([(p / scale).clamp(-448, 448).to(t) for p in x.split(4096)])
        got.append(x if case["layout"] == "nhd" else x.transpose(1, 2))
    return got


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    s = dict(case=case)
    scales = (KEY_SCALE, VALUE_SCALE) if case["cache"] == "e4m3" else (1.0, 1.0)
    s["scales"] = scales
    dim, heads = case["dim"], case["kv_heads"]
    if case["kind"] == "append":
        n, x = case["tokens"], TYPES[case["x"]]
        pages = -(-(n + n // 8 + 64) // case["page"])
        s["k"], s["v"] = _cache(g, pages, case, dev)
        # queries, keys and values are slices of one projection
        every = torch.randn(n, (case["q_heads"] + 2 * heads) * dim, generator=g, device=dev, dtype=torch.float32).to(x)
        cut = case["q_heads"] * dim
        s["xq"] = every[:, :cut].unflatten(1, (case["q_heads"], dim))
        s["xk"] = every[:, cut:cut + heads * dim].unflatten(1, (heads, dim))
        s["xv"] = every[:, cut + heads * dim:].unflatten(1, (heads, dim))
        s["q_out"] = torch.empty(n, case["q_heads"], dim, dtype=x, device=dev)
        s["slots"] = torch.randperm(pages * case["page"], generator=g, device=dev)[:n].to(torch.int32)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device=dev, dtype=torch.int32)
        s["turns"], s["factor"] = _turns(case, dev)
    else:
        rows, used = _pages(case)
        width = max(1, -(-case["length"] // case["page"]))
        more = -(-case["keep"] // case["page"]) if case["kind"] == "evict" else 0
        total = used + more * case["seqs"] + 8
        order = torch.randperm(total, generator=g, device=dev).to(torch.int32)
        table = torch.full((case["seqs"], width), -1, dtype=torch.int32)
        for i, r in enumerate(rows):
            table[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
        table = table.to(dev)
        s["table"] = torch.where(table >= 0, order[table.clamp(min=0).long()], -1).contiguous()
        s["lengths"] = torch.tensor(lengths_of(case), dtype=torch.int32, device=dev)
        s["k"], s["v"] = _cache(g, total, case, dev)
        if case["kind"] == "decode":
            x = TYPES[case["x"]]
            # twice the usual spread: some tokens matter much more than others
            s["q"] = (2 * torch.randn(case["seqs"], case["q_heads"], dim, generator=g, device=dev)).to(x)
            s["scale"] = 1 / math.sqrt(dim)
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(case["seqs"], case["q_heads"], dtype=torch.float32, device=dev)
            s["weight"] = None
            if case["weight"]:
                s["weight"] = torch.rand(case["seqs"], heads, width * case["page"], generator=g, device=dev)
        else:
            w = torch.exp(2 * torch.randn(case["seqs"], heads, width * case["page"], generator=g, device=dev))
            s["weight"] = w * (torch.rand(w.shape, generator=g, device=dev) > 0.2)      # a fifth was never looked at
            s["new_table"] = order[used:used + more * case["seqs"]].reshape(case["seqs"], more).contiguous()
            s["index"] = torch.empty(case["seqs"], heads, case["keep"], dtype=torch.int32, device=dev)
            s["new_weight"] = torch.empty_like(s["weight"])
            s["new_lengths"] = torch.empty(case["seqs"], dtype=torch.int32, device=dev)
    if own:
        from paper_2502_04677_b200 import binding as K
        s["cache"] = K.KvCache(s["k"], s["v"], *scales)
        if case["kind"] == "append":
            s["rope"] = K.kv_rope_table(case["rot"], device=dev, interleaved=case["interleaved"], **_scaling(case))
        elif case["kind"] == "decode":
            s["workspace"] = K.kv_decode_workspace(s["cache"], case["seqs"], case["q_heads"], s["table"].shape[1], case["weight"])
    return s


def _scaling(case):
    """The scaling for long contexts as the framework's call names it: eight times the length of 8,192 that was trained on."""
    if case["scaling"] == "none":
        return dict(theta=10_000.0)
    return dict(theta=10_000.0, scaling=case["scaling"], factor=8.0, original_len=8192)


def _turns(case, dev):
    """Turns per position of every pair, in 64 bits, and the factor on the rotated values."""
    rot, theta, factor = case["rot"], 10_000.0, 8.0
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    if case["scaling"] == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2 * i / rot) / (2 * math.pi)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "yarn":
        ramp = ((8192 * f - 1) / (32 - 1)).clamp(0, 1)
        return f * (ramp + (1 - ramp) / factor), 0.1 * math.log(factor) + 1
    return f, 1.0


def run(s):
    case = s["case"]
    if own:
        return _own(s)
    return {"append": _append, "decode": _decode, "evict": _evict}[case["kind"]](s)


def _own(s):
    from paper_2502_04677_b200 import binding as K
    case = s["case"]
    if case["kind"] == "append":
        K.kv_rope_append(s["cache"], s["xk"], s["xv"], s["slots"], positions=s["positions"], rope=s["rope"], q=s["xq"], q_out=s["q_out"])
        return dict(q=s["q_out"], k=s["k"], v=s["v"])
    if case["kind"] == "decode":
        K.kv_decode(s["cache"], s["q"], s["table"], s["lengths"], s["out"], scale=s["scale"], window=case["window"], lse=s["lse"],
                    weight=s["weight"], workspace=s["workspace"])
        return dict(out=s["out"], lse=s["lse"], weight=s["weight"])
    K.kv_evict(s["cache"], s["weight"], s["table"], s["lengths"], s["new_table"], case["keep"], sinks=case["sinks"], recent=case["recent"],
               index=s["index"], new_weight=s["new_weight"], new_lengths=s["new_lengths"])
    return dict(k=s["k"], v=s["v"], index=s["index"], weight=s["new_weight"], lengths=s["new_lengths"])


def _rotate(x, cos, sin, case):
    rot = case["rot"]
    x, rest = x[..., :rot].float(), x[..., rot:].float()
    if case["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)
    a, b = x[..., :rot // 2], x[..., rot // 2:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)


def _store(x, scale, t):
    if t == torch.float8_e4m3fn:
        return (x / scale).clamp(-448, 448).to(t)
    return x.to(t)


def _put(cache, page, at, x):
    if cache.dtype == torch.float8_e4m3fn:
        cache, x = cache.view(torch.uint8), x.view(torch.uint8)
    cache[page, at] = x


def _append(s):
    case = s["case"]
    turns = s["positions"].double()[:, None] * s["turns"]
    angle = 2 * math.pi * (turns - turns.round())
    cos, sin = ((f(angle) * s["factor"]).float()[:, None] for f in (torch.cos, torch.sin))
    s["q_out"].copy_(_rotate(s["xq"], cos, sin, case))
    slots = s["slots"].long()
    page, at = slots // case["page"], slots % case["page"]
    _put(s["k"], page, at, _store(_rotate(s["xk"], cos, sin, case), s["scales"][0], s["k"].dtype))
    _put(s["v"], page, at, _store(s["xv"].float(), s["scales"][1], s["v"].dtype))
    return dict(q=s["q_out"], k=s["k"], v=s["v"])


def _rows(cache, table, scale):
    """The rows [sequence, token, head, dim] that a page table names, in 32 bits."""
    if cache.dtype == torch.float8_e4m3fn:
        got = cache.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * scale
    else:
        got = cache[table].float()
    return got.flatten(1, 2)


def _decode(s):
    case = s["case"]
    table = s["table"].clamp(min=0).long()
    n, heads, dim = case["seqs"], case["kv_heads"], case["dim"]
    k = _rows(s["k"], table, s["scales"][0]).permute(0, 2, 3, 1)                         # sequence, head, dim, token
    t = torch.arange(k.shape[-1], device=k.device)
    length = s["lengths"].long()[:, None]
    there = (t < length) & (t >= length - (case["window"] or 1 << 40))
    q = s["q"].float().reshape(n, heads, -1, dim)
    score = (q @ k * s["scale"]).masked_fill(~there[:, None, None], -math.inf)
    del k
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    s["lse"].copy_((top + torch.log(total)).reshape(n, -1))
    p = torch.where(total > 0, p / total, 0.0)
    v = _rows(s["v"], table, s["scales"][1]).permute(0, 2, 1, 3)
    s["out"].copy_((p @ v).reshape(n, -1, dim))
    if s["weight"] is not None:
        s["weight"] += p.sum(2)
    return dict(out=s["out"], lse=s["lse"], weight=s["weight"])


def _evict(s):
    case = s["case"]
    page, keep = case["page"], case["keep"]
    w, length = s["weight"], s["lengths"].long()[:, None]
    t = torch.arange(w.shape[-1], device=w.device)
    there = t < length
    held = there & ((t < case["sinks"]) | (t >= length - case["recent"]))
    rank = torch.where(there[:, None], torch.where(held[:, None], math.inf, w), -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    count = length.clamp(max=keep)                                                       # [sequences, 1]
    j = torch.arange(keep, device=w.device)
    some = (j < count)[:, None].expand(best.shape)
    index = torch.where(some, best, w.shape[-1]).sort(-1).values                         # in order of position
    s["index"].copy_(torch.where(some, index, -1))
    s["new_lengths"].copy_(count[:, 0])
    from_ = index.clamp(max=w.shape[-1] - 1)
    s["new_weight"].zero_()
    s["new_weight"][..., :keep] = torch.where(some, w.gather(-1, from_), 0.0)
    b, h, at = some.nonzero(as_tuple=True)
    src, old, new = from_[b, h, at], s["table"].long(), s["new_table"].long()
    for c in (s["k"], s["v"]):
        c = c.view(torch.uint8) if c.dtype == torch.float8_e4m3fn else c
        c[new[b, at // page], at % page, h] = c[old[b, src // page], src % page, h]
    return dict(k=s["k"], v=s["v"], index=s["index"], weight=s["new_weight"], lengths=s["new_lengths"])


def work(case):
    size = {"bf16": 2, "f16": 2, "e4m3": 1}
    heads, dim, c = case["kv_heads"], case["dim"], size[case["cache"]]
    if case["kind"] == "append":
        n, x = case["tokens"], 2
        return dict(bytes=n * (2 * case["q_heads"] * dim * x + 2 * heads * dim * (x + c) + 8),
                    flops=n * (case["q_heads"] + heads) * case["rot"] * 3)
    lengths = lengths_of(case)
    if case["kind"] == "decode":
        seen = [min(n, case["window"] or n) for n in lengths]
        rows = sum(seen)
        # a page that several sequences share is read once
        if shared_pages(case) and not case["window"]:
            lead = shared_pages(case) * case["page"]
            for i in range(0, case["seqs"], 8):
                part = [min(n, lead) for n in lengths[i:i + 8]]
                rows -= sum(part) - max(part)
        b = rows * heads * dim * c * 2 + sum(-(-n // case["page"]) for n in seen) * 4
        b += case["seqs"] * (case["q_heads"] * (dim * 4 + 4) + 4)
        if case["weight"]:
            b += sum(seen) * heads * 8
        return dict(bytes=b, flops=4 * sum(seen) * case["q_heads"] * dim)
    kept = sum(min(n, case["keep"]) for n in lengths)
    width = -(-case["length"] // case["page"]) * case["page"]
    return dict(bytes=kept * heads * dim * c * 4 + sum(lengths) * heads * 4 + case["seqs"] * heads * (width + case["keep"]) * 4,
                flops=sum(lengths) * heads)


def exact(case, seed):
    """The definitions in 64 bits, one sequence (one token) after the other."""
    s = prepare(case, seed)
    ks, vs = s["scales"]
    if case["kind"] == "append":
        return _exact_append(s, case, ks, vs)
    lengths, table = lengths_of(case), s["table"].cpu()
    heads, dim, page = case["kv_heads"], case["dim"], case["page"]
    if case["kind"] == "decode":
        group = case["q_heads"] // heads
        out = torch.zeros(case["seqs"], case["q_heads"], dim, dtype=torch.float64, device="cuda")
        lse = torch.full((case["seqs"], case["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
        weight = s["weight"].double() if case["weight"] else None
        for i, n in enumerate(lengths):
            if n == 0:
                continue
            lo = max(0, n - case["window"]) if case["window"] else 0
            token = torch.arange(lo, n)
            slot = table[i, token // page].long() * page + token % page
            pg, at = (slot // page).cuda(), (slot % page).cuda()
            for h in range(heads):
                kk, vv = (_bytes(c, h, pg, at).double() * f for c, f in ((s["k"], ks), (s["v"], vs)))
                q = s["q"][i, h * group:(h + 1) * group].double()
                z = torch.einsum("gd,td->gt", q, kk) * s["scale"]
                norm = torch.logsumexp(z, 1)
                p = torch.exp(z - norm[:, None])
                out[i, h * group:(h + 1) * group] = torch.einsum("gt,td->gd", p, vv)
                lse[i, h * group:(h + 1) * group] = norm
                if weight is not None:
                    weight[i, h, lo:n] += p.sum(0)
        return dict(out=out, lse=lse, weight=weight)
    k, v = s["k"], s["v"]
    index = torch.full(s["index"].shape, -1, dtype=torch.int64)
    new_w = torch.zeros(s["weight"].shape, dtype=torch.float64)
    w, new = s["weight"].cpu(), s["new_table"].cpu()
    for i, n in enumerate(lengths):
        m = min(n, case["keep"])
        if m == 0:
            continue
        fixed = set(range(min(case["sinks"], n))) | set(range(max(0, n - case["recent"]), n))
        for h in range(heads):
            row = w[i, h, :n].tolist()
            order = sorted(range(n), key=lambda t: (t not in fixed, -row[t], t))
            kept = torch.tensor(sorted(order[:m]))
            index[i, h, :m] = kept
            new_w[i, h, :m] = w[i, h, kept].double()
            j = torch.arange(m)
            for c in (k, v):
                c = c.view(torch.uint8) if c.dtype == torch.float8_e4m3fn else c
                c[new[i, j // page].long().cuda(), (j % page).cuda(), h] = c[table[i, kept // page].long().cuda(), (kept % page).cuda(), h]
    return dict(k=k.double(), v=v.double(), index=index, weight=new_w, lengths=torch.tensor([min(n, case["keep"]) for n in lengths]))


def _bytes(c, h, page, at):
    if c.dtype == torch.float8_e4m3fn:
        return c.view(torch.uint8)[page, at, h].view(torch.float8_e4m3fn)
    return c[page, at, h]


def _exact_append(s, case, ks, vs):
    rot, n = case["rot"], case["tokens"]
    half = rot // 2
    first = [2 * i if case["interleaved"] else i for i in range(half)]
    second = [2 * i + 1 if case["interleaved"] else i + half for i in range(half)]
    # e^(i angle), from whole turns taken off before the angle is formed
    turn = torch.remainder(s["positions"].double().unsqueeze(1) * s["turns"].unsqueeze(0), 1.0)
    unit = torch.polar(torch.full_like(turn, float(s["factor"])), 2 * math.pi * turn)

    def turned(x):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * unit.unsqueeze(1)
        y[..., first], y[..., second] = z.real, z.imag
        return y

    got = dict(q=turned(s["xq"]), k=s["k"].double(), v=s["v"].double())
    at = s["slots"].long()
    page, at = torch.div(at, case["page"], rounding_mode="floor"), torch.remainder(at, case["page"])
    got["k"][page, at] = (turned(s["xk"]) / ks)
    got["v"][page, at] = (s["xv"].double() / vs)
    return got
