"""What the KV-cache calls refuse on the host, before anything is enqueued (no GPU: the pointers are never looked at)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20             # stands for an aligned pointer


@pytest.fixture(scope="module")
def K():
    from paper_2502_04677_b200 import build
    build.build()
    from paper_2502_04677_b200 import binding
    return binding


def cache(K, **change):
    d = dict(k=P, v=P, dtype=K.KV_BF16, n_pages=10, page_size=16, n_heads=2, head_dim=64, k_scale=1.0, v_scale=1.0,
             k_stride=(2048, 128, 64), v_stride=(2048, 128, 64))
    d.update(change)
    d["k_stride"], d["v_stride"] = ((ctypes.c_int64 * 3)(*d[n]) for n in ("k_stride", "v_stride"))
    return K.kv_cache(*[d[n] for n, _ in K.kv_cache._fields_])


def rows(K, heads, dtype=None, data=P, stride=(1024, 64)):
    return K.kv_rows(data, K.KV_BF16 if dtype is None else dtype, heads, (ctypes.c_int64 * 2)(*stride))


BAD_CACHES = [dict(k=None), dict(v=None), dict(dtype=0), dict(dtype=7), dict(n_pages=0), dict(page_size=0), dict(page_size=12), dict(n_heads=0),
              dict(head_dim=0), dict(head_dim=60), dict(k=P + 8), dict(v=P + 2), dict(k_stride=(2048, 32, 64)), dict(v_stride=(2044, 128, 64)),
              dict(k_scale=0.5), dict(dtype=3, k_scale=0.0), dict(dtype=3, v_scale=float("inf")), dict(dtype=3, v_scale=float("nan")),
              dict(dtype=3, head_dim=40), dict(k_stride=(0, 128, 64))]
LARGE_CACHES = [dict(head_dim=320), dict(page_size=1 << 17), dict(n_pages=1 << 30)]


def at(x):
    return ctypes.addressof(x) if x is not None else None


def decode(K, c, q=None, out=None, n=3, table=P, table_stride=8, max_pages=8, lengths=P, scale=0.1, window=0, lse=None, weight=None, ws=None,
           work=P, work_bytes=1 << 40):
    ws = (ctypes.c_int64 * 2)(*ws) if ws else None
    q, out = q or rows(K, 4), out or rows(K, 4, data=2 * P)
    return K.lib().kv_decode(at(c), at(q), at(out), n, table, table_stride, max_pages, lengths, scale, window, lse, weight,
                             at(ws), work, work_bytes, None)


def append(K, c, rope=None, pos=P, slots=P, n=3, q=None, q_out=None, k=None, v=None):
    keep = [k or rows(K, 2), v or rows(K, 2)]
    return K.lib().kv_rope_append(at(c), at(rope), pos, slots, n, at(q), at(q_out), at(keep[0]), at(keep[1]), None)


def evict(K, c, weight=2 * P, ws=(256, 128), n=3, table=P, table_stride=8, max_pages=8, lengths=P, new=P, new_stride=2, new_pages=2, keep=20, sinks=2,
          recent=4, index=P, nw=P, nws=(256, 128), new_len=128, new_lengths=P):
    a, b = ((ctypes.c_int64 * 2)(*x) if x else None for x in (ws, nws))
    return K.lib().kv_evict(at(c), weight, at(a), n, table, table_stride, max_pages, lengths, new, new_stride, new_pages, keep, sinks, recent, index, nw,
                            at(b), new_len, new_lengths, None)


def test_every_declared_call_is_exported(K):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "klpm_kv.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(kv_[a-z_]+)\s*\(", text))
    assert names == set(K.KV_EXPORTS)
    for name in names:
        assert hasattr(K.lib(), name) and hasattr(K, name), name


@pytest.mark.parametrize("change", BAD_CACHES, ids=str)
def test_bad_caches(K, change):
    c = cache(K, **change)
    assert decode(K, c) == K.RT_ERR_INVALID
    assert append(K, c) == K.RT_ERR_INVALID
    assert evict(K, c) == K.RT_ERR_INVALID
    assert K.lib().kv_decode_workspace(at(c), 3, 4, 8, 0) == K.RT_ERR_INVALID


@pytest.mark.parametrize("change", LARGE_CACHES, ids=str)
def test_caches_too_large(K, change):
    c = cache(K, **change)
    assert decode(K, c) == append(K, c) == evict(K, c) == K.RT_ERR_TOO_LARGE


def test_null_cache(K):
    assert decode(K, None) == append(K, None) == evict(K, None) == K.RT_ERR_INVALID


def test_decode_refusals(K):
    c = cache(K)
    inf = float("inf")
    for bad in [dict(n=-1), dict(max_pages=-1), dict(window=-1), dict(scale=float("nan")), dict(scale=inf), dict(q=rows(K, 3)), dict(q=rows(K, 4, K.KV_F32)),
                dict(q=rows(K, 4, K.KV_F16), out=rows(K, 4, K.KV_F16)), dict(out=rows(K, 2)), dict(out=rows(K, 4, K.KV_F16)), dict(q=rows(K, 4, data=P + 1)),
                dict(q=rows(K, 4, data=None)), dict(q=rows(K, 4, data=2 * P)), dict(table=None), dict(lengths=None), dict(table_stride=7), dict(weight=P), dict(work=None),
                dict(work=P + 16), dict(work_bytes=1)]:
        assert decode(K, c, **bad) == K.RT_ERR_INVALID, bad
    assert decode(K, c, max_pages=1 << 27, table_stride=1 << 27) == K.RT_ERR_TOO_LARGE
    assert decode(K, c, n=1 << 17) == K.RT_ERR_TOO_LARGE
    one = cache(K, n_heads=1, k_stride=(1024, 64, 64), v_stride=(1024, 64, 64))
    assert K.lib().kv_decode_workspace(at(one), 65535, 65535, 1 << 26, 1) == K.RT_ERR_TOO_LARGE
    assert decode(K, c, n=0) == K.RT_OK
    need = K.lib().kv_decode_workspace(at(c), 3, 4, 8, 1)
    assert need > 0 and decode(K, c, weight=P, ws=(256, 128), work_bytes=need - 1) == K.RT_ERR_INVALID
    assert K.lib().kv_decode_workspace(at(c), -1, 4, 8, 0) == K.lib().kv_decode_workspace(at(c), 3, 3, 8, 0) == K.RT_ERR_INVALID


def test_append_refusals(K):
    c = cache(K)
    rope = lambda dim=64, turns=P: K.kv_rope(turns, dim, 0, 1.0)
    for bad in [dict(n=-1), dict(slots=None), dict(k=rows(K, 3)), dict(v=rows(K, 1)), dict(v=rows(K, 2, K.KV_F16)), dict(k=rows(K, 2, K.KV_F16), v=rows(K, 2, K.KV_F16)),
                dict(q=rows(K, 4)), dict(q_out=rows(K, 4)), dict(q=rows(K, 4), q_out=rows(K, 3)), dict(q=rows(K, 4), q_out=rows(K, 4, K.KV_F16)),
                dict(q=rows(K, 4), q_out=rows(K, 4, stride=(2048, 64))), dict(rope=rope(66)), dict(rope=rope(0)), dict(rope=rope(7)), dict(rope=rope(64, None)),
                dict(rope=rope(), pos=None), dict(k=rows(K, 2, data=P + 1)), dict(k=rows(K, 2, K.KV_E4M3), v=rows(K, 2, K.KV_E4M3))]:
        assert append(K, c, **bad) == K.RT_ERR_INVALID, bad
    assert append(K, c, n=0) == K.RT_OK


def test_evict_refusals(K):
    c = cache(K)
    for bad in [dict(n=-1), dict(max_pages=-1), dict(new_pages=1), dict(keep=0), dict(keep=33), dict(sinks=-1), dict(recent=-1), dict(sinks=17), dict(new_len=19),
                dict(table_stride=7), dict(new_stride=1), dict(ws=None), dict(nws=None), dict(weight=None), dict(table=None), dict(lengths=None), dict(new=None),
                dict(index=None), dict(nw=None), dict(nw=2 * P), dict(new_lengths=None)]:
        assert evict(K, c, **bad) == K.RT_ERR_INVALID, bad
    assert evict(K, c, max_pages=1 << 27, table_stride=1 << 27) == K.RT_ERR_TOO_LARGE
    assert evict(K, c, n=0) == K.RT_OK


def test_rope_table_refusals(K):
    f = lambda turns=P, dim=64, theta=1e4, kind=0, scale=1.0, length=8192.0, fast=32.0, slow=1.0: K.lib().kv_rope_table(
        turns, dim, theta, kind, scale, length, fast, slow, None, None)
    for bad in [dict(turns=None), dict(dim=0), dict(dim=5), dict(theta=0.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(kind=4), dict(kind=-1),
                dict(kind=1, scale=0.5), dict(kind=2, scale=float("nan")), dict(kind=2, scale=2.0, dim=2), dict(kind=3, scale=2.0, length=0.0),
                dict(kind=3, scale=2.0, fast=1.0), dict(kind=3, scale=2.0, slow=-1.0)]:
        assert f(**bad) == K.RT_ERR_INVALID, bad
    assert f(dim=512) == K.RT_ERR_TOO_LARGE


def test_prefix_slots_refuses_a_missing_tree(K):
    assert K.lib().rt_prefix_slots(None, P, P, 1, P, 4, 4, None) == K.RT_ERR_INVALID


def test_the_binding_refuses_cpu_tensors(K):
    import torch
    x = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        K.KvCache(x, x)


def test_the_binding_refuses_numbers_that_do_not_fit(K):
    for x in (-1, 1 << 31, 1 << 40):
        with pytest.raises(ValueError):
            K._count(x, "window")
    assert K._count((1 << 31) - 1, "window") == (1 << 31) - 1


def test_outputs_whose_rows_overlap_are_refused(K):
    """Expanded outputs and others that share memory between rows: two rows would be written (or added to) at the same time."""
    c = cache(K)
    for stride in [(0, 64), (1024, 0), (1024, 63), (64, 64), (128, 64), (255, 64), (-128, 64), (96, 64), (0, 0), (64, 128), (1 << 62, 32)]:
        assert decode(K, c, out=rows(K, 4, data=2 * P, stride=stride)) == K.RT_ERR_INVALID, stride
        assert append(K, c, q=rows(K, 4), q_out=rows(K, 4, data=2 * P, stride=stride)) == K.RT_ERR_INVALID, stride
        assert append(K, c, q=rows(K, 4, stride=stride), q_out=rows(K, 4, stride=stride)) == K.RT_ERR_INVALID, stride
    for ws in [(0, 128), (256, 0), (255, 128), (128, 128), (256, 127), (0, 0), (127, 1 << 40)]:         # rows of 8 pages of 16 tokens
        assert decode(K, c, weight=P, ws=ws) == K.RT_ERR_INVALID, ws
    for nws in [(0, 128), (256, 0), (200, 128), (128, 128), (0, 0)]:
        assert evict(K, c, nws=nws) == K.RT_ERR_INVALID, nws
