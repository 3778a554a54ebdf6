"""Both kernels of kv_decode in every instance, with and without weights and windows, against a plain implementation in 64 bits.

A row is a sequence, a cache head and up to 16 of its query heads (8 for heads above 128 elements).  The kernel of small calls takes a call only while there
are at most 296 rows (148 for heads above 128 elements or more than 8 query heads per cache head) and, with weights, only if all query heads of a cache
head are in one row.  The bounds are those of test_gpu_kv.py, formed for all heads of a sequence at once."""
import math

import pytest
import torch

from test_gpu_kv import BF, E4, HALF, HF, K, TINY, U, fill_, gen, make_cache, tables, values

pytestmark = pytest.mark.gpu

MOST_ROWS = 296

PAIRS = [(BF, BF), (HF, HF), (BF, E4), (HF, E4)]
# elements of a head, query heads per cache head, rows of a cache head
SIZES = [(64, 5, 1), (48, 12, 1), (128, 8, 1), (112, 16, 1), (96, 17, 2), (64, 40, 3), (192, 8, 1), (256, 5, 1), (160, 9, 2), (256, 17, 3)]


def plain(c, q, table, lengths, scale, window, weight):
    n, qh, dim = q.shape
    heads, group, page = c.n_heads, qh // c.n_heads, c.page_size
    out = torch.zeros(n, qh, dim, dtype=torch.float64, device="cuda")
    lse = torch.full((n, qh), -math.inf, dtype=torch.float64, device="cuda")
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    if weight is not None:
        weight = weight.double()
        weight_tol = 4 * U * weight
    for b, length in enumerate(lengths):
        t = torch.arange(max(0, length - window) if window else 0, length, device="cuda")
        if len(t) == 0:
            continue
        slots = table[b].long()[t // page] * page + t % page
        k, v = values(c.k, slots, c.c.k_scale), values(c.v, slots, c.c.v_scale)
        x = q[b].double().reshape(heads, group, dim)
        s = torch.einsum("hgd,thd->hgt", x, k) * scale
        size = (torch.einsum("hgd,thd->hgt", x.abs(), k.abs()) * abs(scale)).amax(-1)
        norm = torch.logsumexp(s, -1)
        p = torch.exp(s - norm[..., None])
        o = torch.einsum("hgt,thd->hgd", p, v)
        spread = torch.einsum("hgt,thd->hgd", p, v.abs())
        ds = (2 * dim + 4) * U * size + dim * 2.0 ** -39 * x.abs().amax(-1) * k.abs().amax((0, 2))[:, None] * abs(scale)
        dp = 2 * ds + (2 * len(t) + 16) * U + 4 * U * s.abs().amax(-1)
        out[b], lse[b] = o.reshape(qh, dim), norm.reshape(qh)
        tol = (dp + 2.0 ** -16 + 2 * len(t) * U)[..., None] * spread + len(t) * 2.0 ** -39 * v.abs().amax((0, 2))[:, None, None]
        out_tol[b] = tol.reshape(qh, dim) + HALF[q.dtype] * out[b].abs() + TINY[q.dtype]
        lse_tol[b] = dp.reshape(qh) + 4 * U * lse[b].abs()
        if weight is not None:
            weight[b][:, t] += p.sum(1)
            weight_tol[b][:, t] += (p * (dp + 4 * U)[..., None]).sum(1) + 4 * U * weight[b][:, t]
    return out, lse, weight, out_tol, lse_tol, weight_tol if weight is not None else None


def check(c, q, table, lengths, window, with_weight):
    n, qh, dim = q.shape
    w = torch.rand(n, c.n_heads, table.shape[1] * c.page_size, generator=gen(5), device="cuda") if with_weight else None
    out, lse, weight, out_tol, lse_tol, weight_tol = plain(c, q, table, lengths, dim ** -0.5, window, w)
    got, got_lse = torch.full_like(q, 7.0), torch.full((n, qh), 7.0, device="cuda")
    K().kv_decode(c, q, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), got, window=window, lse=got_lse, weight=w)
    assert ((got.double() - out).abs() <= out_tol).all()
    none = lse == -math.inf
    assert torch.equal(none, got_lse == -math.inf) and (got[none] == 0).all()
    assert ((got_lse.double() - lse).abs()[~none] <= lse_tol[~none]).all()
    if w is not None:
        assert ((w.double() - weight).abs() <= weight_tol).all()


def nan_elsewhere(c, table, lengths, window):
    """NaN in all that no sequence attends to."""
    mine = torch.zeros(c.n_pages * c.page_size, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lengths):
        t = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        mine[table[b].long()[t // c.page_size] * c.page_size + t % c.page_size] = True
    for x in (c.k, c.v):
        fill_(x, (~mine).nonzero()[:, 0], math.nan)


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("dim,group,rows", SIZES)
@pytest.mark.parametrize("tq,tc", PAIRS, ids=str)
def test_every_instance(tq, tc, dim, group, rows, large):
    lengths = [300, 1, 0, 130, 77]
    heads = MOST_ROWS // (len(lengths) * rows) + 1 if large else 2
    assert (len(lengths) * heads * rows > MOST_ROWS) == large and (large or len(lengths) * heads * rows <= 148)
    for window in (0, 1, 50):
        g = gen(dim + group + window)
        table, pages = tables(g, lengths, 16)
        c = make_cache(g, pages, 16, heads, dim, tc, "nhd", (0.0625, 0.03125) if tc == E4 else (1.0, 1.0))
        nan_elsewhere(c, table, lengths, window)
        q = (2 * torch.randn(len(lengths), heads * group, dim, generator=g, device="cuda")).to(tq)
        for with_weight in (False, True):
            check(c, q, table, lengths, window, with_weight)


@pytest.mark.parametrize("window", [0, 333])
@pytest.mark.parametrize("group", [4, 16, 20])
@pytest.mark.parametrize("tc", [BF, E4], ids=str)
def test_many_rows_that_are_cut(tc, group, window):
    """More rows than the kernel of small calls takes, cut among warps wherever their spans end; windows that begin inside a tile."""
    g = gen(31)
    lengths = [(1999, 0, 37, 640, 1001)[i % 5] for i in range(160)]
    table, pages = tables(g, lengths, 8)
    c = make_cache(g, pages, 8, 2, 128, tc, "hnd")
    nan_elsewhere(c, table, lengths, window)
    q = torch.randn(len(lengths), 2 * group, 128, generator=g, device="cuda").to(BF)
    assert len(lengths) * 2 > MOST_ROWS
    for with_weight in (False, True):
        check(c, q, table, lengths, window, with_weight)


@pytest.mark.parametrize("group", [9, 33])
def test_few_long_rows_of_several_groups_of_heads(group):
    """Without weights one cluster per row, with them rows that many warps join."""
    g = gen(37)
    lengths = [4001, 130]
    for dim in (64, 192):
        table, pages = tables(g, lengths, 16)
        c = make_cache(g, pages, 16, 1, dim, HF)
        q = torch.randn(2, group, dim, generator=g, device="cuda").to(HF)
        for window in (0, 1500):
            for with_weight in (False, True):
                check(c, q, table, lengths, window, with_weight)
