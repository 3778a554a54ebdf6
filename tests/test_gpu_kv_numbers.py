"""Numbers at the ends of their types in the KV-cache operators.  The plain implementations and the bounds are those of test_gpu_kv.py."""
import math
from fractions import Fraction

import pytest
import torch

from test_gpu_kv import BF, E4, HALF, HF, K, TINY, U, check_decode, fill_, gen, make_cache, tables, values, wide_table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [3, 12])
@pytest.mark.parametrize("power", [126, 121, -110, -126])
def test_queries_at_the_ends_of_bf16_next_to_an_8_bit_cache(power, group):
    """Every finite query has a power of two that makes it f16: the largest, 2^128 less one step, and the smallest normal ones."""
    g = gen(13)
    table, pages = tables(g, [300, 17], 16)
    c = make_cache(g, pages, 16, 1, 64, E4, "nhd", (0.0625, 0.0625))
    lens = torch.tensor([300, 17], dtype=torch.int32, device="cuda")
    f = 2.0 ** power
    q = (torch.randn(2, group, 64, generator=g, device="cuda").clamp(-3.9, 3.9) * f).to(BF)
    if power == 126:
        q[0, 0, 5], q[1, 2, 63] = torch.finfo(BF).max, -torch.finfo(BF).max
    check_decode(c, q, table, lens, scale=0.25 / f)
    check_decode(c, q, table, lens, scale=0.25 / f, weight=False)


def decode_with_what_is_not_finite(c, q, table, lengths, scale):
    """Outputs in 64 bits and bounds of their errors (those of plain_decode, element by element); a token whose score is -inf takes no part."""
    n, qh, dim = q.shape
    group, page = qh // c.n_heads, c.page_size
    out, tol = (torch.zeros(n, qh, dim, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, length in enumerate(lengths):
        t = torch.arange(length, device="cuda")
        slots = table[b].long()[t // page] * page + t % page
        kk, vv = values(c.k, slots, 1.0), values(c.v, slots, 1.0)
        for h in range(qh):
            g, x = h // group, q[b, h].double()
            s = kk[:, g] @ x * scale
            part = s != -math.inf
            if not part.any():
                continue
            k, v, s = kk[part, g], vv[part, g], s[part]
            p = torch.softmax(s, 0)
            size = (k.abs() @ x.abs() * abs(scale)).max()
            out[b, h] = (p[:, None] * v).sum(0)
            finite = torch.where(v.isfinite(), v, 0.0).abs()
            dp = 2 * (2 * dim + 4) * U * size + (2 * len(v) + 16) * U + 4 * U * s.abs().max()
            tol[b, h] = (dp + 2.0 ** -16 + 2 * len(v) * U) * (p @ finite) + len(v) * 2.0 ** -39 * finite.amax(0) + HALF[q.dtype] * out[b, h].abs() + TINY[q.dtype]
    return out, tol


def same_or_near(got, want, tol):
    plain = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.double()[want.isinf()], want[want.isinf()])
    assert ((got.double() - want).abs()[plain] <= tol[plain]).all()


# rows x cache heads decide how many warps join a row in the kernels of large calls: 32 (16), 8, 1
@pytest.mark.parametrize("seqs,heads", [(3, 2), (33, 2), (80, 2)])
@pytest.mark.parametrize("group,dim", [(3, 64), (12, 80), (2, 200)])
@pytest.mark.parametrize("t", [BF, HF], ids=str)
def test_infinities_and_nan_among_the_values(t, group, dim, seqs, heads):
    g = gen(17 + dim)
    lens = [(700, 61, 5, 130)[i % 4] for i in range(seqs)]
    table, pages = tables(g, lens, 8)
    c = make_cache(g, pages, 8, heads, dim, t)
    q = torch.rand(seqs, heads * group, dim, generator=g, device="cuda").to(t)       # (positive: a key of -inf has a score of -inf)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    at = lambda b, i: (int(table[b, i // 8]), i % 8)
    for b, n in enumerate(lens):
        kind = b % 9
        last, mid = at(b, n - 1), at(b, n // 2)
        if kind == 0:
            c.v[last][:, 3] = math.inf
        elif kind == 1:
            c.v[last][0, 1::2], c.v[mid][0, 1::3] = math.inf, -math.inf              # one sign, the other, both
        elif kind == 2:
            c.v[mid] = math.nan
        elif kind == 3:
            c.k[mid], c.v[mid] = -math.inf, math.nan                                 # takes no part: the rest counts
        elif kind == 4:
            c.k[mid], c.v[mid], c.v[last][:, 5:9] = -math.inf, math.inf, -math.inf
        elif kind == 5:
            c.v[at(b, 0)][:, dim - 1], c.v[last][:, dim - 1], c.v[last][:, 0] = math.nan, math.inf, math.inf
        elif kind == 6:
            c.k[at(b, 0)][heads - 1], c.v[at(b, 0)][heads - 1, ::2], c.v[mid][heads - 1, ::5] = -math.inf, math.nan, math.inf
        elif kind == 7:
            for i in range(n):
                c.v[at(b, i)][:, 2] = math.inf if i % 2 else 1.0
    want, tol = decode_with_what_is_not_finite(c, q, table, lens, dim ** -0.5)
    assert want.isnan().any() and want.isinf().any() and want.isfinite().any()
    for pages in (table, wide_table(table, 8)):
        out = torch.full_like(q, 7.0)
        K().kv_decode(c, q, pages, lengths, out)
        same_or_near(out, want, tol)


def test_an_infinite_value_counts_however_small_its_probability():
    c = make_cache(gen(3), 4, 16, 1, 64, BF)
    c.k.fill_(1.0)
    c.k[1, 4], c.v[1, 4] = -60.0, math.inf               # a score of -480: e^-488 is 0 in 32 bits
    q = torch.ones(1, 2, 64, dtype=BF, device="cuda")
    table, lens = torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"), torch.tensor([40], dtype=torch.int32, device="cuda")
    for pages in (table, wide_table(table, 16)):
        out = torch.zeros_like(q)
        K().kv_decode(c, q, pages, lens, out)
        assert (out == math.inf).all()


@pytest.mark.parametrize("tc,seqs,length", [(BF, 1, 20_000), (BF, 2, 131_072), (E4, 2, 131_072), (HF, 200, 2000)], ids=str)
def test_a_nan_value_does_not_make_a_call_slow(tc, seqs, length):
    """One NaN among the values, at the end of a row: the call takes a few times what it takes without.  (Walking such a row token by token takes a thousand
    times as long; 25 leaves room for whatever else the machine does.)"""
    g = gen(19)
    table, pages = tables(g, [length] * seqs, 16)
    c = make_cache(g, pages, 16, 2, 128, tc)
    q = torch.randn(seqs, 16, 128, generator=g, device="cuda").to(tc if tc != E4 else BF)
    lens = torch.full((seqs,), length, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    work = K().kv_decode_workspace(c, seqs, 16, table.shape[1])

    def best():
        times = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            K().kv_decode(c, q, table, lens, out, workspace=work)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    best()
    clean = best()
    assert out.isfinite().all()
    fill_(c.v, (table.long()[:1, -1] * 16 + (length - 1) % 16), math.nan)
    bad = best()
    assert out[0].isnan().all() and out[1:].isfinite().all()
    print("%s %d x %d: %.1f us, with a NaN %.1f us" % (tc, seqs, length, clean * 1e3, bad * 1e3))
    assert bad < 25 * clean


def test_outputs_whose_rows_lie_apart_in_any_order():
    """Heads before sequences, and rows that fill one another's gaps: what is refused is memory shared by two rows, not an unusual layout."""
    g = gen(23)
    lens = [90, 33, 7]
    table, pages = tables(g, lens, 16)
    c = make_cache(g, pages, 16, 2, 64, BF)
    q = torch.randn(3, 2, 64, generator=g, device="cuda").to(BF)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want, want_w = torch.empty_like(q), torch.zeros(3, 2, table.shape[1] * 16, device="cuda")
    K().kv_decode(c, q, table, lengths, want, weight=want_w)
    width = want_w.shape[2]
    for s0, s1 in ((64, 3 * 64), (2 * 64, 3 * 64), (3 * 64, 64), (70, 300)):
        room = torch.full((600,), 9.0, dtype=BF, device="cuda")
        out = room.as_strided((3, 2, 64), (s0, s1, 1))
        w = torch.zeros(9 * width, device="cuda").as_strided((3, 2, width), (s0 * width // 64, s1 * width // 64, 1))
        turned = room.clone().as_strided((3, 2, 64), (s0, s1, 1))
        K().kv_decode(c, q, table, lengths, out, weight=w)
        K().kv_rope_append(c, q, q, torch.full((3,), -1, dtype=torch.int32, device="cuda"), q=q, q_out=turned)
        assert torch.equal(out, want) and torch.equal(w, want_w) and torch.equal(turned, q)
        out.fill_(9.0)
        assert (room == 9).all()


@pytest.mark.parametrize("rot", [16, 128])
def test_far_positions_against_exact_turns(rot):
    """Positions up to the ends of 31 bits, whole turns taken off in rational arithmetic.  The kernel's product in 64 bits is off by half a step, at 2^31 positions
    of 1 / (2 pi) turns 2^-25 of a turn, its rest in 32 bits by 2^-26 more, and sine and cosine by 2 ulp: the angle by less than 2^-24 of a turn, 2 pi
    2^-24 or 6.3 u; two products and a sum, with the factors' errors, 6 u."""
    rope = K().kv_rope_table(rot, theta=10_000.0, device="cuda")
    positions = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, 1_500_000_001, 987_654_321, -77, 1 << 20, 0]
    n, turns = len(positions), [Fraction(x) for x in rope.turns.tolist()]
    exact = torch.tensor([[float((p * f) % 1) for f in turns] for p in positions], dtype=torch.float64, device="cuda")[:, None] * (2 * math.pi)
    q = torch.randn(n, 3, rot, generator=gen(41), device="cuda")
    c = make_cache(gen(1), 4, 4, 1, rot, BF)
    got = torch.empty_like(q)
    K().kv_rope_append(c, q[:, :1], q[:, :1], torch.full((n,), -1, dtype=torch.int32, device="cuda"),
                       positions=torch.tensor(positions, dtype=torch.int32, device="cuda"), rope=rope, q=q, q_out=got)
    a, b = q.double()[..., :rot // 2], q.double()[..., rot // 2:]
    want = torch.cat([a * exact.cos() - b * exact.sin(), a * exact.sin() + b * exact.cos()], -1)
    size = (a.abs() + b.abs()).repeat(1, 1, 2)
    assert ((got.double() - want).abs() <= 13 * U * size).all()
