"""The KV-cache operators against plain implementations in 64 bits, through the public binding.

Tolerances (derived, not tuned): a stored value is off by at most half a step of its type, HALF[t] relative (plus half the smallest
subnormal).  Before that, 32-bit arithmetic: u = 2^-24 per operation; a dot product or sum of n terms is off by at most 2 n u times the sum of
the terms' absolute values (2: partial sums of the tensor cores may be cut off instead of rounded).
"""
import itertools
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
HALF = {torch.float32: 2.0 ** -24, BF: 2.0 ** -8, HF: 2.0 ** -11, E4: 2.0 ** -4}
TINY = {torch.float32: 2.0 ** -150, BF: 2.0 ** -134, HF: 2.0 ** -25, E4: 2.0 ** -10}
U = 2.0 ** -24


def K():
    from paper_2502_04677_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make_cache(g, pages, page, heads, dim, t, layout="nhd", scales=(1.0, 1.0)):
    mem = (pages, page, heads, dim) if layout == "nhd" else (pages, heads, page, dim)
    got = []
    for s in scales:
        x = torch.randn(mem, generator=g, device="cuda")
        x = (x / s).clamp(-448, 448).to(t) if t == E4 else x.to(t)
        got.append(x if layout == "nhd" else x.transpose(1, 2))
    return K().KvCache(got[0], got[1], *scales)


def values(c, slots, scale):
    """[slots, heads, dim] in 64 bits."""
    p, a = slots // c.shape[1], slots % c.shape[1]
    if c.dtype == E4:
        return c.contiguous().view(torch.uint8)[p, a].view(E4).double() * scale
    return c[p, a].double() * scale


def fill_(c, slots, value):
    """Writes `value` into whole slots."""
    if c.dtype == E4:
        c = c.view(torch.uint8)
        value = 0x7f
    c[slots // c.shape[1], slots % c.shape[1]] = value


# ---------------------------------------------------------------------------------------------------------------- append

def plain_rope(x, positions, rope, rot, interleaved):
    x = x.double().clone()
    turn = torch.remainder(positions.double()[:, None] * rope.turns, 1.0)
    c, s = torch.cos(2 * math.pi * turn)[:, None] * rope.factor, torch.sin(2 * math.pi * turn)[:, None] * rope.factor
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    xa, xb = x[..., a], x[..., b]
    size = torch.zeros_like(x)
    size[..., a] = size[..., b] = xa.abs() + xb.abs()
    x[..., a], x[..., b] = xa * c - xb * s, xa * s + xb * c
    return x, size * rope.factor


APPEND = [
    # n, q heads, heads, dim, rot, interleaved, x, cache, page, layout, scaling
    (1, 4, 1, 64, 64, False, BF, BF, 1, "nhd", "none"),
    (7, 6, 2, 128, 128, True, HF, HF, 16, "hnd", "linear"),
    (33, 8, 8, 80, 40, False, BF, BF, 8, "nhd", "ntk"),
    (33, 5, 5, 80, 40, True, BF, E4, 8, "nhd", "yarn"),
    (40, 2, 1, 256, 96, False, torch.float32, HF, 4, "hnd", "yarn"),
    (40, 3, 3, 192, 192, True, torch.float32, E4, 64, "nhd", "none"),
    (19, 2, 2, 16, 2, False, torch.float32, BF, 2, "nhd", "linear"),
    (1500, 7, 3, 64, 32, True, HF, E4, 32, "hnd", "ntk"),
    (2049, 3, 1, 128, 128, False, BF, BF, 16, "nhd", "yarn"),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
@pytest.mark.parametrize("sliced", [False, True])
def test_append(case, sliced):
    n, qh, h, dim, rot, inter, tx, tc, page, layout, scaling = case
    g = gen(n + dim)
    scales = (0.125, 0.3) if tc == E4 else (1.0, 1.0)
    c = make_cache(g, n // page + 9, page, h, dim, tc, layout, scales)
    before = [x.clone() for x in (c.k, c.v)]
    wide = torch.randn(n, qh + 2 * h, dim, generator=g, device="cuda") * 3
    x = wide.to(tx)
    if sliced:      # rows that start anywhere and lie far apart
        room = torch.zeros(n, qh + 2 * h, dim + 3, dtype=tx, device="cuda")
        room[..., 1:dim + 1] = x
        x = room[..., 1:dim + 1]
    q, k, v = x[:, :qh], x[:, qh:qh + h], x[:, qh + h:]
    rope = K().kv_rope_table(rot, theta=500_000.0, interleaved=inter, scaling=scaling, factor=4.0 if scaling != "none" else 1.0, original_len=4096)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 2 ** 31 - 1 if n > 1 else 0
    if n > 4:
        pos[1], pos[2] = -5, 0
    slots = torch.randperm((n // page + 9) * page, generator=g, device="cuda")[:n].to(torch.int32)
    if n > 6:
        slots[3], slots[4], slots[5] = -1, (n // page + 9) * page, 2 ** 31 - 1
    q_out = torch.full((n, qh, dim), 7.0, dtype=tx, device="cuda")
    K().kv_rope_append(c, k, v, slots, positions=pos, rope=rope, q=q, q_out=q_out)
    # two products, a sum, and cos and sin (2 ulp each) of an angle that is off by 2^-23 of a turn at most: under 16 u of |a| + |b|
    want, size = plain_rope(q, pos, rope, rot, inter)
    assert ((q_out.double() - want).abs() <= HALF[tx] * want.abs() + TINY[tx] + 16 * U * size).all()
    there = (slots >= 0) & (slots < (n // page + 9) * page)
    s = slots[there].long()
    for new, old, src, scale, turned in ((c.k, before[0], k, scales[0], True), (c.v, before[1], v, scales[1], False)):
        want, size = plain_rope(src, pos, rope, rot, inter) if turned else (src.double(), torch.zeros_like(src, dtype=torch.float64))
        want, size = want[there] / scale, size[there] / scale
        if tc == E4:
            want = want.clamp(-448, 448)
        got = values(new, s, 1.0)
        assert ((got - want).abs() <= HALF[tc] * (1 + 2 * U) * want.abs() + TINY[tc] + (16 * U + U) * size + U * want.abs()).all()
        rest = torch.ones((n // page + 9) * page, dtype=torch.bool, device="cuda")
        rest[s] = False
        rest = rest.nonzero()[:, 0]
        assert torch.equal(values(new, rest, 1.0), values(old, rest, 1.0))
    # in place, and without rotation
    q2 = q.clone()
    K().kv_rope_append(c, k, v, slots, positions=pos, rope=rope, q=q2, q_out=q2)
    assert torch.equal(q2, q_out)
    K().kv_rope_append(c, k, v, slots)
    if tc == tx:
        assert torch.equal(values(c.k, s, 1.0), k[there].double())


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
@pytest.mark.parametrize("rot", [4, 64, 128])
def test_rope_table(scaling, rot):
    factor = 1.0 if scaling == "none" else 8.0
    rope = K().kv_rope_table(rot, theta=10_000.0, scaling=scaling, factor=factor, original_len=8192)
    for i, got in enumerate(rope.turns.tolist()):
        theta = 1e4 * factor ** (rot / (rot - 2)) if scaling == "ntk" else 1e4
        f = theta ** (-2 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            r = 8192 * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (r - 1) / (32 - 1)))
            f = keep * f + (1 - keep) * f / factor
        assert abs(got - f / (2 * math.pi)) <= 1e-13 * f
    assert rope.factor == pytest.approx(0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0, rel=1e-6)


def test_append_8_bit_values_that_do_not_fit():
    c = make_cache(gen(1), 4, 4, 1, 16, E4)
    x = torch.tensor([1e9, -1e9, math.inf, -math.inf, math.nan, 448.0, 464.0, -0.0] * 2, device="cuda").reshape(1, 1, 16)
    K().kv_rope_append(c, x, x, torch.tensor([5], dtype=torch.int32, device="cuda"))
    got = values(c.k, torch.tensor([5], device="cuda"), 1.0).flatten().tolist()
    assert got[:4] == [448, -448, 448, -448] and math.isnan(got[4]) and got[5:8] == [448, 448, 0]


# ---------------------------------------------------------------------------------------------------------------- decode

def plain_decode(c, q, table, lengths, scale, window, weight):
    """out, lse, weight and bounds of their errors, sequence by sequence in 64 bits."""
    n, qh, dim = q.shape
    group, page = qh // c.n_heads, c.page_size
    out = torch.zeros(n, qh, dim, dtype=torch.float64, device="cuda")
    lse = torch.full((n, qh), -math.inf, dtype=torch.float64, device="cuda")
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    weight = weight.double() if weight is not None else None
    weight_tol = torch.zeros_like(weight) if weight is not None else None
    for b in range(n):
        length = min(max(int(lengths[b]), 0), table.shape[1] * page)
        t = torch.arange(max(0, length - window) if window else 0, length, device="cuda")
        pg = table[b].long()[t // page]
        t = t[(pg >= 0) & (pg < c.n_pages)]
        if len(t) == 0:
            continue
        slots = table[b].long()[t // page] * page + t % page
        kk, vv = values(c.k, slots, c.c.k_scale), values(c.v, slots, c.c.v_scale)
        for h in range(qh):
            g = h // group
            x = q[b, h].double()
            s, size = kk[:, g] @ x * scale, kk[:, g].abs() @ x.abs() * abs(scale)
            m = s.max()
            if m == -math.inf:
                continue
            p = torch.exp(s - m)
            total = p.sum()
            p = p / total
            out[b, h] = p @ vv[:, g]
            lse[b, h] = m + torch.log(total)
            # scores: a dot product of dim terms, two more products; a weight: exp of a difference of two such (3 ulp), its sum over len(t)
            # and the division; its product with a value: probabilities are used with at least 16 bits, and like the elements of a
            # query next to an 8-bit cache not below 2^-39 of the largest
            ds = (2 * dim + 4) * U * size.max() + dim * 2.0 ** -39 * (x.abs().max() * kk[:, g].abs().max() * abs(scale))
            dp = 2 * ds + (2 * len(t) + 16) * U + 4 * U * s.abs().max()
            out_tol[b, h] = (dp + 2.0 ** -16 + 2 * len(t) * U) * (p @ vv[:, g].abs()) + len(t) * 2.0 ** -39 * vv[:, g].abs().max() + HALF[q.dtype] * out[b, h].abs() + TINY[q.dtype]
            lse_tol[b, h] = dp + 4 * U * lse[b, h].abs()
            if weight is not None:
                weight[b, g, t] += p
                weight_tol[b, g, t] += p * (dp + 4 * U)
    if weight is not None:
        weight_tol += 4 * U * weight.abs()
    return out, lse, weight, out_tol, lse_tol, weight_tol


def check_decode(c, q, table, lengths, scale=None, window=0, weight=True, **more):
    n, qh, dim = q.shape
    g = gen(5)
    w = torch.rand(n, c.n_heads, table.shape[1] * c.page_size, generator=g, device="cuda") if weight else None
    scale = dim ** -0.5 if scale is None else scale
    out, lse, weight, out_tol, lse_tol, weight_tol = plain_decode(c, q, table, lengths, scale, window, w)
    got = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    got_lse = torch.full((n, qh), 7.0, device="cuda")
    K().kv_decode(c, q, table, lengths, got, scale=scale, window=window, lse=got_lse, weight=w, **more)
    assert ((got.double() - out).abs() <= out_tol).all()
    none = lse == -math.inf
    assert torch.equal(none, got_lse == -math.inf)
    assert ((got_lse.double() - lse).abs()[~none] <= lse_tol[~none]).all()
    if w is not None:
        assert ((w.double() - weight).abs() <= weight_tol).all()
    # the same with room for many more tokens in the table (other kernels take it): lengths beyond the narrow one's end are cut off by hand
    lengths = lengths.clamp(max=table.shape[1] * c.page_size)
    wide = wide_table(table, c.page_size)
    w2 = torch.rand(n, c.n_heads, wide.shape[1] * c.page_size, generator=g, device="cuda") if weight is not None else None
    before = w2.clone() if w2 is not None else None
    got2, lse2 = torch.full_like(got, 7.0), torch.full_like(got_lse, 7.0)
    K().kv_decode(c, q, wide, lengths, got2, scale=scale, window=window, lse=lse2, weight=w2, **more)
    assert ((got2.double() - out).abs() <= out_tol).all()
    assert torch.equal(none, lse2 == -math.inf)
    assert ((lse2.double() - lse).abs()[~none] <= lse_tol[~none]).all()
    if w2 is not None:
        k = table.shape[1] * c.page_size
        assert torch.equal(w2[..., k:], before[..., k:])
        added = (weight - torch.rand(n, c.n_heads, k, generator=gen(5), device="cuda").double())
        assert ((w2[..., :k].double() - before[..., :k].double() - added).abs() <= weight_tol + 4 * U * w2[..., :k].double()).all()
    return got, got_lse, w


def wide_table(table, page):
    return torch.cat([table, torch.full((table.shape[0], 40_000 // page), -1, dtype=torch.int32, device="cuda")], 1)


def tables(g, lengths, page, width=None, spare=3):
    """Pages in any order; -1 where there is none.  Returns the table and the number of pages."""
    need = [-(-max(x, 0) // page) for x in lengths]
    width = max(1, max(need)) if width is None else width
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
    used = 0
    for i, x in enumerate(need):
        table[i, :x] = order[used:used + x]
        used += x
    return table, total


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 1000]
DECODE = [
    # q heads, heads, dim, page, layout, q, cache
    (1, 1, 16, 1, "nhd", BF, BF),
    (8, 1, 64, 16, "nhd", BF, BF),
    (8, 8, 80, 8, "hnd", BF, BF),
    (6, 2, 128, 16, "nhd", HF, HF),
    (32, 8, 128, 64, "hnd", BF, BF),
    (34, 2, 128, 1, "nhd", BF, BF),
    (16, 1, 128, 4, "nhd", HF, HF),
    (40, 1, 96, 16, "nhd", BF, BF),
    (9, 3, 192, 32, "nhd", HF, HF),
    (10, 2, 256, 2, "hnd", BF, BF),
    (18, 2, 256, 16, "nhd", HF, HF),
    (8, 2, 64, 1, "nhd", BF, E4),
    (8, 2, 128, 16, "hnd", HF, E4),
    (20, 1, 128, 64, "nhd", BF, E4),
    (5, 5, 80, 16, "nhd", HF, E4),
    (8, 1, 256, 16, "hnd", BF, E4),
    (17, 1, 48, 8, "nhd", BF, E4),
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
@pytest.mark.parametrize("window", [0, 1, 50])
def test_decode(case, window):
    qh, h, dim, page, layout, tq, tc = case
    g = gen(dim + qh)
    table, pages = tables(g, LENGTHS, page)
    c = make_cache(g, pages, page, h, dim, tc, layout, (0.0625, 0.03125) if tc == E4 else (1.0, 1.0))
    q = (2 * torch.randn(len(LENGTHS), qh, dim, generator=g, device="cuda")).to(tq)
    lengths = torch.tensor(LENGTHS, dtype=torch.int32, device="cuda")
    # what no sequence has a right to read: NaN
    mine = torch.zeros(pages * page, dtype=torch.bool, device="cuda")
    for b, n in enumerate(LENGTHS):
        t = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        mine[table[b].long()[t // page] * page + t % page] = True
    for x in (c.k, c.v):
        fill_(x, (~mine).nonzero()[:, 0], math.nan)
    check_decode(c, q, table, lengths, window=window)


@pytest.mark.parametrize("tc", [BF, E4], ids=str)
@pytest.mark.parametrize("seqs,length,window", [(1, 9001, 0), (2, 5003, 0), (3, 20_011, 4097), (70, 777, 0), (1, 4096, 4096)])
def test_decode_split_over_the_length(tc, seqs, length, window):
    g = gen(length)
    lens = [max(0, length - 97 * i) for i in range(seqs)]
    table, pages = tables(g, lens, 16, width=length // 16 + 40)
    c = make_cache(g, pages, 16, 2, 128, tc)
    q = torch.randn(seqs, 10, 128, generator=g, device="cuda").to(BF) * 3
    check_decode(c, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), window=window)


def test_decode_pages_that_are_not_there():
    g = gen(3)
    lens = [64, 64, 200, 200, 33, 9999, -3]
    table, pages = tables(g, [64, 64, 200, 200, 33, 200, 200], 8)
    table[1] = -1                                       # nothing at all
    table[2, 3], table[2, 24] = -1, pages               # holes
    table[3, ::2] = 2 ** 31 - 1
    table[4, :4] = -(2 ** 31)
    c = make_cache(g, pages, 8, 2, 64, BF)
    q = torch.randn(7, 8, 64, generator=g, device="cuda").to(BF)
    out, lse, _ = check_decode(c, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all() and (out[6] == 0).all()
    check_decode(c, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), window=9)


def test_decode_large_scores_and_equal_keys():
    g = gen(8)
    table, pages = tables(g, [500, 500], 16)
    c = make_cache(g, pages, 16, 1, 64, BF)
    q = torch.randn(2, 4, 64, generator=g, device="cuda").to(BF) * 200        # one token takes all of a row's weight
    check_decode(c, q, table, torch.tensor([500, 499], dtype=torch.int32, device="cuda"))
    check_decode(c, q, table, torch.tensor([500, 499], dtype=torch.int32, device="cuda"), scale=-1.0)
    check_decode(c, q * 0, table, torch.tensor([500, 499], dtype=torch.int32, device="cuda"))
    check_decode(c, q, table, torch.tensor([500, 499], dtype=torch.int32, device="cuda"), scale=0.0)


@pytest.mark.parametrize("tq,tc", [(BF, BF), (HF, HF), (BF, E4), (HF, E4)], ids=str)
def test_decode_small_and_large_queries(tq, tc):
    """Elements far apart in size keep their products."""
    g = gen(9)
    table, pages = tables(g, [300, 17], 16)
    c = make_cache(g, pages, 16, 1, 64, tc, "nhd", (0.0625, 0.0625) if tc == E4 else (1.0, 1.0))
    big, small = (2.0 ** 100, 2.0 ** -100) if tq == BF else (2.0 ** 11, 2.0 ** -10)
    lens = torch.tensor([300, 17], dtype=torch.int32, device="cuda")
    for f in (big, small):
        q = (torch.randn(2, 3, 64, generator=g, device="cuda") * f).to(tq)
        check_decode(c, q, table, lens, scale=0.125 / f)
    q = torch.randn(2, 3, 64, generator=g, device="cuda").to(tq)
    q[:, :, 5] *= 2.0 ** 9
    check_decode(c, q, table, lens, scale=0.01)


def test_decode_infinities_and_nan_in_what_is_attended_to():
    g = gen(4)
    table, pages = tables(g, [40] * 4, 8)
    c = make_cache(g, pages, 8, 1, 64, BF)
    q = torch.ones(4, 2, 64, device="cuda", dtype=BF)
    lens = torch.full((4,), 40, dtype=torch.int32, device="cuda")
    at = lambda b, t: (int(table[b, t // 8]), t % 8)
    c.k[at(0, 13)] = -math.inf                  # a score of -inf: that token has no weight
    c.k[at(1, 13)] = math.nan
    c.v[at(2, 13)] = math.inf
    c.v[at(3, 2)][..., 7] = -math.inf           # one element only
    for pages in (table, wide_table(table, 8)):
        w = torch.zeros(4, 1, pages.shape[1] * 8, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(4, 2, device="cuda")
        K().kv_decode(c, q, pages, lens, out, lse=lse, weight=w)
        w = w[:, :, :40]
        assert w[0, 0, 13] == 0 and torch.isfinite(out[0]).all() and torch.isfinite(lse[0]).all()
        assert abs(float(w[0].sum()) - 2) < 1e-4
        assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all() and torch.isnan(w[1]).all()
        assert (out[2] == math.inf).all() and torch.isfinite(lse[2]).all()
        assert (out[3, :, 7] == -math.inf).all() and torch.isfinite(out[3, :, :7]).all() and torch.isfinite(out[3, :, 8:]).all()
    c.k[at(3, 0)[0]] = -math.inf                # a whole sequence of scores of -inf: nothing to attend to
    for pages in (table, wide_table(table, 8)):
        K().kv_decode(c, q, pages, torch.full((4,), 8, dtype=torch.int32, device="cuda"), out, lse=lse)
        assert (out[3] == 0).all() and (lse[3] == -math.inf).all()


def test_decode_strides_and_rows_that_start_anywhere():
    g = gen(6)
    lens = [100, 37, 5]
    table, pages = tables(g, lens, 16)
    c = make_cache(g, pages, 16, 2, 64, BF)
    room = torch.randn(3, 5, 70, generator=g, device="cuda").to(BF)
    q = room[:, 1:5, 3:67]
    wide = torch.full((3, 20), -7, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = check_decode(c, q, table, lengths)
    o = torch.full((3, 5, 70), 9.0, device="cuda", dtype=BF)
    w = torch.rand(3, 5, 300, generator=gen(5), device="cuda")
    before = w.clone()
    K().kv_decode(c, q, wide[:, :table.shape[1]], lengths, o[:, 1:5, 3:67], weight=w[:, 1:5:2, 3:])
    assert torch.equal(o[:, 1:5, 3:67], want[0])
    o[:, 1:5, 3:67] = 9
    assert (o == 9).all()
    changed = (w != before).nonzero()
    assert set(changed[:, 1].tolist()) <= {1, 3} and int(changed[:, 2].min()) >= 3 and int(changed[:, 2].max()) < 103


def test_decode_the_same_every_time_and_under_a_graph():
    g = gen(11)
    lens = [3001, 17, 0, 999]
    table, pages = tables(g, lens, 16, width=400)
    c = make_cache(g, pages, 16, 4, 128, BF)
    q = torch.randn(4, 16, 128, generator=g, device="cuda").to(BF)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    first = check_decode(c, q, table, lengths)
    out, lse, w = torch.empty_like(q), torch.empty(4, 16, device="cuda"), torch.zeros(4, 4, 6400, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                K().kv_decode(c, q, table, lengths, out, lse=lse, weight=w)
            graphs.append(graph)
    torch.cuda.synchronize()
    seen = []
    for step in range(4):
        w.zero_()
        out.fill_(5)
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        seen.append((out.clone(), lse.clone(), w.clone()))
    assert all(torch.equal(a, b) for s in seen[1:] for a, b in zip(s, seen[0]))
    assert torch.equal(seen[0][0], first[0]) and torch.equal(seen[0][1], first[1])
    # other lengths under the same graph
    lengths.copy_(torch.tensor([5, 6400, 3000, 0], dtype=torch.int32))
    table.copy_(torch.where(table < 0, table[0, 0], table))
    graphs[0].replay()
    torch.cuda.synchronize()
    got = (out.clone(), lse.clone())
    want = check_decode(c, q, table, lengths)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("wide", [False, True])
def test_decode_on_two_streams(wide):
    g = gen(12)
    cases = []
    for i, n in enumerate((2500, 4000)):
        table, pages = tables(g, [n, n // 2], 16)
        c = make_cache(g, pages, 16, 2, 64, BF)
        q = torch.randn(2, 8, 64, generator=g, device="cuda").to(BF)
        table = wide_table(table, 4) if wide else table          # (160,000 tokens)
        cases.append((c, q, table, torch.tensor([n, n // 2], dtype=torch.int32, device="cuda")))
    want = []
    for c, q, table, lens in cases:
        out = torch.empty_like(q)
        K().kv_decode(c, q, table, lens, out)
        ref, _, _, tol, _, _ = plain_decode(c, q, table, lens, q.shape[2] ** -0.5, 0, None)
        assert ((out.double() - ref).abs() <= tol).all()
        want.append(out)
    outs = [[torch.empty_like(x[1]) for _ in range(20)] for x in cases]
    weights = [torch.zeros(2, 2, x[2].shape[1] * 16, device="cuda") for x in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for k in range(20):
        for s, x, o, w in zip(streams, cases, outs, weights):
            with torch.cuda.stream(s):
                K().kv_decode(*x, o[k], weight=w)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for got, w in zip(outs, want) for o in got)
    for w, x in zip(weights, cases):                             # every call added 1 for each of a cache head's four heads
        assert ((w.double().sum(-1) - 20 * 4).abs() <= 20 * 4 * 1e-4).all()


FIRST_CALL = """
import torch
from paper_2502_04677_b200 import binding as K
k, v = (torch.randn(300, 16, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
c = K.KvCache(k, v)
q = torch.randn(3, 8, 64, device="cuda").to(torch.bfloat16)
lens = torch.tensor([4000, 17, 300], dtype=torch.int32, device="cuda")
new = torch.arange(280, 286, dtype=torch.int32, device="cuda").reshape(3, 2)
x = torch.randn(3, 2, 64, device="cuda").to(torch.bfloat16)
slots = torch.tensor([4700, 4701, 4702], dtype=torch.int32, device="cuda")
turned = torch.empty_like(q)
rope = K.kv_rope_table(64)
got = []
for pages in (250, 2500):
    table = torch.arange(pages, dtype=torch.int32, device="cuda").remainder(250).repeat(3, 1)
    out, lse = torch.empty_like(q), torch.empty(3, 8, device="cuda")
    w, nw = torch.zeros(3, 2, pages * 16, device="cuda"), torch.empty(3, 2, 40, device="cuda")
    index, nl = torch.empty(3, 2, 32, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    def call():
        K.kv_rope_append(c, x, x, slots, positions=lens, rope=rope, q=q, q_out=turned)
        K.kv_decode(c, turned, table, lens, out, lse=lse, weight=w)
        K.kv_evict(c, w, table, lens, new, 32, sinks=2, recent=8, index=index, new_weight=nw, new_lengths=nl)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    graph.replay()
    torch.cuda.synchronize()
    seen = [t.clone() for t in (out, lse, w, index, nw, nl)]
    w.zero_()
    call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(seen, (out, lse, w, index, nw, nl)))
    assert torch.isfinite(out).all() and nl.tolist() == [32, 17, 32]
print("first calls captured")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    got = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "first calls captured" in got.stdout, got.stderr[-2000:]


def test_decode_empty_calls():
    c = make_cache(gen(1), 4, 4, 1, 64, BF)
    none = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    K().kv_decode(c, none, torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), none.clone())
    q = torch.randn(2, 2, 64, device="cuda").to(BF)
    out, lse = torch.full_like(q, 3), torch.full((2, 2), 3.0, device="cuda")
    K().kv_decode(c, q, torch.empty(2, 0, dtype=torch.int32, device="cuda"), torch.tensor([4, 0], dtype=torch.int32, device="cuda"), out, lse=lse,
                  weight=torch.empty(2, 1, 0, device="cuda"))
    assert (out == 0).all() and (lse == -math.inf).all()


def test_a_cache_of_more_than_four_gigabytes():
    """Byte offsets beyond 32 bits, at both ends of a page."""
    pages, page, h, dim = 70_000, 16, 16, 128
    c = K().KvCache(*(torch.zeros(pages, page, h, dim, dtype=BF, device="cuda") for _ in range(2)))
    g = gen(2)
    table = torch.tensor([[pages - 1, 0, pages - 2, 40_000]], dtype=torch.int32, device="cuda")
    slots = (table.long()[0][:, None] * page + torch.arange(page, device="cuda")).flatten().to(torch.int32)
    k, v = (torch.randn(64, h, dim, generator=g, device="cuda").to(BF) for _ in range(2))
    K().kv_rope_append(c, k, v, slots)
    q = torch.randn(1, 32, dim, generator=g, device="cuda").to(BF)
    check_decode(c, q, table, torch.tensor([64], dtype=torch.int32, device="cuda"))
    assert torch.equal(c.k[table[0].long()].reshape(64, h, dim), k)
    index, nw, nl = torch.empty(1, h, 16, dtype=torch.int32, device="cuda"), torch.empty(1, h, 16, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    K().kv_evict(c, torch.rand(1, h, 64, generator=g, device="cuda"), table, torch.tensor([64], dtype=torch.int32, device="cuda"),
                 torch.tensor([[69_000]], dtype=torch.int32, device="cuda"), 16, index=index, new_weight=nw, new_lengths=nl)
    for head in range(h):
        assert torch.equal(c.v[69_000, :, head], v[index[0, head].long(), head])


# ---------------------------------------------------------------------------------------------------------------- evict

def check_evict(c, w, table, lengths, keep, sinks, recent, width=None, new_table=None):
    n, h, page = len(lengths), c.n_heads, c.page_size
    new_pages = -(-keep // page)
    if new_table is None:
        new_table = torch.arange(c.n_pages - n * new_pages, c.n_pages, dtype=torch.int32, device="cuda").reshape(n, new_pages)
    width = w.shape[2] if width is None else width
    before = [x.clone() for x in (c.k, c.v)]
    index = torch.full((n, h, keep), 9, dtype=torch.int32, device="cuda")
    nw = torch.full((n, h, width), 9.0, device="cuda")
    nl = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    K().kv_evict(c, w, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), new_table, keep, sinks=sinks, recent=recent,
                 index=index, new_weight=nw, new_lengths=nl)
    changed = torch.zeros(c.n_pages * page, dtype=torch.bool, device="cuda")
    rows, pt, ind, nws, nls, nt = w.tolist(), table.tolist(), index.tolist(), nw.cpu(), nl.tolist(), new_table.tolist()
    for b in range(n):
        length = min(max(lengths[b], 0), table.shape[1] * page)
        there = [t for t in range(length) if 0 <= pt[b][t // page] < c.n_pages]
        m = min(keep, len(there))
        assert nls[b] == m
        for g in range(h):
            def rank(t):
                x = rows[b][g][t]
                return (not (t < sinks or t >= length - recent), math.inf if math.isnan(x) else -x, not math.isnan(x) and 0, t)
            kept = sorted(sorted(there, key=lambda t: (rank(t)[0], math.isnan(rows[b][g][t]) and rank(t)[0], rank(t)[1] if rank(t)[0] else 0, t))[:m])
            assert ind[b][g] == kept + [-1] * (keep - m), (b, g)
            want = torch.zeros(width)
            want[:m] = torch.tensor([rows[b][g][t] for t in kept])
            assert torch.equal(nws[b, g].nan_to_num(nan=-77.0), want.nan_to_num(nan=-77.0))
            j = [j for j in range(m) if 0 <= nt[b][j // page] < c.n_pages]
            if not j:
                continue
            j = torch.tensor(j, device="cuda")
            src = torch.tensor(kept, device="cuda")[j]
            s = table[b].long()[src // page] * page + src % page
            d = new_table[b].long()[j // page] * page + j % page
            changed[d] = True
            for x, old in zip((c.k, c.v), before):
                assert torch.equal(values(x, d, 1.0)[:, g], values(old, s, 1.0)[:, g])
    rest = (~changed).nonzero()[:, 0]
    for x, old in zip((c.k, c.v), before):
        assert torch.equal(values(x, rest, 1.0).nan_to_num(nan=-7.0), values(old, rest, 1.0).nan_to_num(nan=-7.0))


EVICT = [
    # lengths, keep, sinks, recent, heads, dim, page, layout, cache
    ([0, 1, 2, 15, 16, 17, 40, 100], 16, 2, 5, 2, 64, 4, "nhd", BF),
    ([1], 1, 0, 0, 1, 16, 1, "nhd", BF),
    ([100, 99], 1, 1, 0, 3, 128, 16, "hnd", HF),
    ([100, 99], 7, 3, 4, 3, 128, 16, "hnd", E4),
    ([2000, 1023, 1024, 1025], 1024, 4, 100, 2, 80, 8, "nhd", BF),
    ([5000], 37, 0, 0, 2, 64, 64, "nhd", E4),
    ([20_011, 9000], 4099, 16, 1000, 1, 64, 16, "hnd", HF),
    ([70_001], 65_000, 0, 1, 2, 16, 32, "nhd", E4),
    ([400_001, 37, 3000], 5000, 3, 100, 1, 16, 64, "nhd", E4),
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(case, kind):
    lengths, keep, sinks, recent, h, dim, page, layout, t = case
    g = gen(keep)
    table, pages = tables(g, lengths, page, spare=len(lengths) * -(-keep // page))
    spare = len(lengths) * -(-keep // page)
    # the pages of `table` are any of all pages: the new ones are those it does not name
    free = torch.ones(pages, dtype=torch.bool, device="cuda")
    free[table[table >= 0].long()] = False
    new = free.nonzero()[:, 0].to(torch.int32)[:spare].reshape(len(lengths), -1)
    c = make_cache(g, pages, page, h, dim, t, layout)
    w = torch.exp(2 * torch.randn(len(lengths), h, table.shape[1] * page, generator=g, device="cuda"))
    if kind == "ties":
        w = w.clamp(max=2).mul(2).floor()
    if kind == "odd":
        pick = torch.rand(w.shape, generator=g, device="cuda")
        for i, x in enumerate((math.inf, -math.inf, math.nan, 0.0, -0.0, -1.0, 1e-42, 3e38)):
            w = torch.where((pick >= i / 16) & (pick < (i + 1) / 16), x, w)
    check_evict(c, w, table, lengths, keep, sinks, recent, new_table=new)


def test_evict_pages_that_are_not_there():
    g = gen(3)
    lens = [64, 64, 200, 9999, -3]
    table, pages = tables(g, [64, 64, 200, 200, 200], 8, spare=40)
    c = make_cache(g, pages, 8, 2, 64, BF)
    free = torch.ones(pages, dtype=torch.bool, device="cuda")
    free[table[table >= 0].long()] = False
    new = free.nonzero()[:, 0].to(torch.int32)[:20].reshape(5, 4).clone()
    table[0] = -1
    table[1, 1:7] = pages
    table[2, ::2], table[3, 0] = -1, 2 ** 31 - 1
    new[2, 1], new[3, 2] = -1, pages
    w = torch.rand(5, 2, table.shape[1] * 8, generator=g, device="cuda")
    check_evict(c, w, table, lens, 30, 4, 6, new_table=new)
    check_evict(c, w, table, lens, 30, 4, 6, width=30, new_table=new)


def test_evict_strides_and_a_graph():
    g = gen(7)
    lens = [500, 300]
    table, pages = tables(g, lens, 16, spare=16)
    c = make_cache(g, pages, 16, 2, 64, BF)
    free = torch.ones(pages, dtype=torch.bool, device="cuda")
    free[table[table >= 0].long()] = False
    new = free.nonzero()[:, 0].to(torch.int32).reshape(2, 8)
    room = torch.rand(2, 5, 600, generator=g, device="cuda")
    w = room[:, 1:5:2, 3:520]
    check_evict(c, w, table, lens, 100, 4, 6, new_table=new[:, :7])
    out = torch.full((2, 5, 600), 9.0, device="cuda")
    index, nl = torch.empty(2, 2, 100, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    call = lambda: K().kv_evict(c, w, table, lengths, new[:, :7], 100, sinks=4, recent=6, index=index, new_weight=out[:, 1:5:2, 3:203], new_lengths=nl)
    call()
    torch.cuda.synchronize()
    want = (out.clone(), index.clone(), c.k.clone())
    assert (out[:, ::2] == 9).all() and (out[:, :, :3] == 9).all() and (out[:, :, 203:] == 9).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    out.fill_(9)
    index.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(index, want[1]) and torch.equal(c.k, want[2])


# ------------------------------------------------------------------------------------------------- the tree and the cache

def test_prefix_slots_name_the_tokens_of_the_match():
    B = K()
    prompts = [[1, 2, 3, 4, 5, 6, 7], [1, 2, 3, 9], [1, 2, 3, 4, 5, 8, 8, 8], [5], [], [1, 2]]
    tok = torch.tensor([x for p in prompts for x in p], dtype=torch.int32, device="cuda")
    off = torch.tensor([0] + list(itertools.accumulate(len(p) for p in prompts)), dtype=torch.int64, device="cuda")
    for budget in (0, 1000):
        tree = B.rt_build(tok, off, max_nodes=64, max_pool_tokens=512, budget_tokens=budget)
        queries = [[1, 2, 3, 4, 5, 6, 7, 7], [1, 2, 3, 9], [1, 2], [2], [], [5, 5], [1, 2, 3, 4, 5, 8]]
        qt = torch.tensor([x for p in queries for x in p], dtype=torch.int32, device="cuda")
        qo = torch.tensor([0] + list(itertools.accumulate(len(p) for p in queries)), dtype=torch.int64, device="cuda")
        n = len(queries)
        m, node = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        B.rt_match_batch(tree, qt, qo, m, node)
        assert m.tolist() == [7, 4, 2, 0, 0, 1, 6]
        room = torch.full((n, 12), 77, dtype=torch.int32, device="cuda")
        B.rt_prefix_slots(tree, node, m, room[:, :9])
        rows = room.tolist()
        for r, k in zip(rows, m.tolist()):
            assert all(x >= 0 for x in r[:k]) and r[k:9] == [-1] * (9 - k) and r[9:] == [77] * 3
        assert rows[0][:3] == rows[1][:3] and rows[0][:2] == rows[2][:2] and rows[0][:5] == rows[6][:5]
        stored = {}
        for q, r, k in zip(queries, rows, m.tolist()):
            for d in range(k):
                assert stored.setdefault(r[d], (d, tuple(q[:d + 1]))) == (d, tuple(q[:d + 1]))       # one slot, one prefix
        # a narrow row, insertions since the match, nodes that are none
        B.rt_insert(tree, torch.tensor([1, 2, 3, 4, 0], dtype=torch.int32, device="cuda"), torch.tensor([0, 5], dtype=torch.int64, device="cuda"))
        again = torch.zeros(n, 3, dtype=torch.int32, device="cuda")
        B.rt_prefix_slots(tree, node, m, again)
        assert again.tolist() == [r[:3] for r in rows]
        B.rt_prefix_slots(tree, torch.tensor([-5, 0, 10 ** 6, 63, 2, 2, 2], dtype=torch.int32, device="cuda"),
                          torch.tensor([1, 1, 1, 1, 10 ** 9, -4, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), again)
        assert (again == -1).all()
        assert B.rt_sync_status(tree) == 0
        B.rt_destroy(tree)


@pytest.mark.parametrize("budget", [0, 20_000])
def test_a_step_of_an_engine(budget):
    """Prompts are scheduled on the tree; their keys and values live in the slots that the tree hands out; every prompt's next token
    attends to them; then the caches are shortened and attended to again.  Against a dense cache per prompt."""
    B = K()
    from paper_2502_04677_b200 import workloads as W
    w = W.tiny(n_queries=40, n_prefill=60)
    pt, po = (x.cuda() for x in w.prefill.materialize())
    qt, qo = (x.cuda() for x in w.queries.materialize())
    n, h, qh, dim = w.queries.n, 2, 8, 64
    cap = pt.numel() + qt.numel() + 8 * (n + w.prefill.n) + 16
    tree = B.rt_build(pt, po, max_nodes=2 * (n + w.prefill.n) + 16, max_pool_tokens=cap, budget_tokens=max(budget, 0))
    order, unc = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
    ttft = torch.zeros(n, dtype=torch.int64, device="cuda")
    B.klpm_run(tree, qt, qo, w.arrivals.cuda(), B.make_params(B.POLICY_KLPM, 2, 0, 1, w.start_tick), order, unc, ttft)
    assert B.rt_sync_status(tree) == 0
    m, node = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
    B.rt_match_batch(tree, qt, qo, m, node)
    lens = qo.diff().to(torch.int32)
    if budget == 0:
        assert torch.equal(m, lens)             # everything that was processed is cached
    width = int(m.max())
    slots = torch.zeros(n, width, dtype=torch.int32, device="cuda")
    B.rt_prefix_slots(tree, node, m, slots)
    # one slot, one prefix: a slot says which token came last and which slot the one before it has, and the other way round
    after, came_from = {}, {}
    toks, offs = qt.tolist(), qo.tolist()
    for i, row in enumerate(slots.tolist()):
        before = -1
        for d in range(int(m[i])):
            assert 0 <= row[d] < cap
            step = (before, toks[offs[i] + d])
            assert after.setdefault(step, row[d]) == row[d] and came_from.setdefault(row[d], step) == step
            before = row[d]
        assert row[int(m[i]):] == [-1] * (width - int(m[i]))
    # keys and values of a token go by its prefix: here by its slot, as two prompts share a slot exactly where they share the prefix
    g = gen(21)
    ks, vs = (torch.randn(cap, h, dim, generator=g, device="cuda").to(BF) for _ in range(2))
    cache = B.KvCache(*(torch.zeros(cap, 1, h, dim, dtype=BF, device="cuda") for _ in range(2)))
    rope = B.kv_rope_table(dim)
    used = torch.unique(slots[slots >= 0]).long()
    depth = torch.zeros(cap, dtype=torch.int32, device="cuda")
    for i in range(n):
        k = int(m[i])
        depth[slots[i, :k].long()] = torch.arange(k, dtype=torch.int32, device="cuda")
    q = torch.randn(n, qh, dim, generator=g, device="cuda").to(BF)
    turned = torch.empty_like(q)
    B.kv_rope_append(cache, ks[used], vs[used], used.to(torch.int32), positions=depth[used], rope=rope)
    B.kv_rope_append(cache, q[:, :h], q[:, :h], torch.full((n,), -1, dtype=torch.int32, device="cuda"), positions=m, rope=rope, q=q, q_out=turned)
    _, _, weight = check_decode(cache, turned, slots, m)
    # what was attended to is what the prompts' own tokens say, laid out densely
    want, _ = plain_rope(ks[slots[0, :int(m[0])].long()], torch.arange(int(m[0]), device="cuda"), rope, dim, False)
    got = cache.k[slots[0, :int(m[0])].long(), 0].double()
    assert ((got - want).abs() <= HALF[BF] * want.abs() + 1e-5).all()
    # shortened to 100 tokens each, in slots of a second cache area
    big = B.KvCache(*(torch.cat([x, torch.zeros(n * 100, 1, h, dim, dtype=BF, device="cuda")]) for x in (cache.k, cache.v)))
    fresh = (cap + torch.arange(n * 100, dtype=torch.int32, device="cuda")).reshape(n, 100)
    check_evict(big, weight, slots, m.tolist(), 100, 4, 16, new_table=fresh)
    check_decode(big, turned, fresh, torch.minimum(m, torch.tensor(100, device="cuda", dtype=torch.int32)))
    B.rt_destroy(tree)
