"""ctypes binding of libklpm.so: argument marshalling only.

Same names as the C ABI (include/klpm.h; include/klpm_kv.h for the KV cache).  Tensors must live on the CUDA device; every step of the
path runs in the library's kernels.  There is no CPU fallback: importing this module fails if the
library has not been built, and every call fails on a non-CUDA tensor.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("KLPM_LIB") or os.path.join(_HERE, "libklpm.so")

RT_OK, RT_ERR_INVALID, RT_ERR_CAPACITY, RT_ERR_BUDGET, RT_ERR_LIMIT, RT_ERR_CUDA = 0, -1, -2, -3, -4, -5
RT_ERR_TOO_LARGE = -6
SELECT_NOALLOC_MAX_QUERIES = 1 << 22
POLICY_FCFS, POLICY_LPM, POLICY_KLPM = 0, 1, 2
_ERR = {-1: "RT_ERR_INVALID", -2: "RT_ERR_CAPACITY", -3: "RT_ERR_BUDGET", -4: "RT_ERR_LIMIT", -5: "RT_ERR_CUDA",
        -6: "RT_ERR_TOO_LARGE"}


class KlpmError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__("%s returned %s (%d)" % (where, _ERR.get(code, "?"), code))
        self.code = code


class rt_config(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("max_nodes", ctypes.c_int64), ("max_pool_tokens", ctypes.c_int64),
                ("budget_tokens", ctypes.c_int64), ("max_clock", ctypes.c_int64)]


class klpm_params(ctypes.Structure):
    _fields_ = [("policy", ctypes.c_int32), ("k", ctypes.c_int32), ("c_num", ctypes.c_int64),
                ("c_den", ctypes.c_int64), ("start_tick", ctypes.c_int64)]


if not os.path.exists(LIB_PATH):
    raise ImportError("libklpm.so is not built: run `python -m paper_2502_04677_b200.build` "
                      "(there is no CPU fallback for this library)")

_lib = ctypes.CDLL(LIB_PATH)
_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64

_lib.klpm_abi_version.restype = _i32
_lib.rt_create.restype = _i32
_lib.rt_create.argtypes = [ctypes.POINTER(rt_config), ctypes.POINTER(_vp)]
_lib.rt_build.restype = _i32
_lib.rt_build.argtypes = [_vp, _vp, _i32, ctypes.POINTER(rt_config), _vp, ctypes.POINTER(_vp)]
_lib.rt_insert.restype = _i32
_lib.rt_insert.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp]
_lib.rt_match_batch.restype = _i32
_lib.rt_match_batch.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp]
_lib.rt_match_batch_ex.restype = _i32
_lib.rt_match_batch_ex.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp]
_lib.rt_prefix_slots.restype = _i32
_lib.rt_prefix_slots.argtypes = [_vp, _vp, _vp, _i32, _vp, _i64, _i32, _vp]
_lib.rt_stats.restype = _i32
_lib.rt_stats.argtypes = [_vp] + [ctypes.POINTER(_i64)] * 5
_lib.rt_clone.restype = _i32
_lib.rt_clone.argtypes = [_vp, _vp, ctypes.POINTER(_vp)]
_lib.rt_checkpoint.restype = _i32
_lib.rt_checkpoint.argtypes = [_vp, _vp]
_lib.rt_rollback.restype = _i32
_lib.rt_rollback.argtypes = [_vp, _vp]
_lib.rt_status_detail.restype = _i32
_lib.rt_status_detail.argtypes = [_vp, ctypes.POINTER(_i32)]
_lib.rt_sync_status.restype = _i32
_lib.rt_sync_status.argtypes = [_vp, _vp]
_lib.rt_destroy.restype = _i32
_lib.rt_destroy.argtypes = [_vp]
_lib.klpm_select.restype = _i32
_lib.klpm_select.argtypes = [_vp, _vp, _vp, _i32, _i64, ctypes.POINTER(klpm_params), _vp, _vp]
_lib.klpm_select_topk.restype = _i32
_lib.klpm_select_topk.argtypes = [_vp, _vp, _vp, _i32, _i32, _vp, _vp]
_lib.klpm_select_noalloc.restype = _i32
_lib.klpm_select_noalloc.argtypes = [_vp, _vp, _vp, _i32, _i64, ctypes.POINTER(klpm_params), _vp, _vp]
_lib.klpm_replay.restype = _i32
_lib.klpm_replay.argtypes = [_vp, _vp, _i32, _vp, _vp, _vp, _i32, ctypes.POINTER(klpm_params), _vp, _vp, _vp, _vp]
_lib.klpm_run_ex.restype = _i32
_lib.klpm_run_ex.argtypes = [_vp, _vp, _vp, _vp, _i32, ctypes.POINTER(klpm_params), _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.klpm_batch_times.restype = _i32
_lib.klpm_batch_times.argtypes = [_vp, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp]
_lib.klpm_run_last_only_batch.restype = _i32
_lib.klpm_run_last_only_batch.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, ctypes.POINTER(klpm_params), _vp, _vp, _vp, _vp, _vp, _vp]
_lib.rt_debug_counters.restype = _i32
_lib.rt_debug_counters.argtypes = [_vp, ctypes.POINTER(_i64 * 16)]
_lib.klpm_debug_set.restype = _i32
_lib.klpm_debug_set.argtypes = [ctypes.c_char_p, _i64]
_lib.klpm_run_path.restype = _i32
_lib.klpm_run_path.argtypes = [_vp]
_lib.klpm_run.restype = _i32
_lib.klpm_run.argtypes = [_vp, _vp, _vp, _vp, _i32, ctypes.POINTER(klpm_params), _vp, _vp, _vp, _vp, _vp]

MATCH_STATE_BYTES = 32

EXPORTS = ["klpm_abi_version", "rt_create", "rt_build", "rt_insert", "rt_match_batch", "rt_match_batch_ex", "rt_prefix_slots", "rt_stats",
           "rt_sync_status", "rt_status_detail", "rt_clone", "rt_checkpoint", "rt_rollback", "rt_destroy", "klpm_select", "klpm_select_topk", "klpm_select_noalloc", "klpm_replay", "klpm_run", "klpm_run_ex", "klpm_run_path", "klpm_batch_times", "klpm_debug_set", "klpm_run_last_only_batch", "rt_debug_counters"]


def lib() -> ctypes.CDLL:
    return _lib


def _dev(t: Optional[torch.Tensor], dtype, name: str, nullable: bool = False) -> Optional[int]:
    if t is None:
        if nullable:
            return None
        raise ValueError("%s must not be None" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (this library has no CPU path)" % name)
    if t.dtype is not dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor" % (name, dtype))
    return t.data_ptr()


def _stream() -> int:
    """The current stream's handle.  (Without a torch.cuda.Stream object around it: that object costs more than the
    launches of a small call.)"""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _table(t: torch.Tensor, name: str):
    """Pointer and row stride of a page table: int32, two dimensions, entries of a row next to one another."""
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (this library has no CPU path)" % name)
    if t.dtype is not torch.int32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be a two-dimensional int32 tensor with contiguous rows" % name)
    return t.data_ptr(), t.stride(0)


def _check(code: int, where: str) -> None:
    if code != RT_OK:
        raise KlpmError(code, where)


def make_params(policy: int, k: int = 1, c_num: int = 0, c_den: int = 1, start_tick: int = 0) -> klpm_params:
    return klpm_params(int(policy), int(k), int(c_num), int(c_den), int(start_tick))


class Tree:
    """Handle of a device radix tree (rt_tree*)."""

    def __init__(self, handle: ctypes.c_void_p, budget_tokens: int = 0):
        self._h = handle
        self.budget_tokens = int(budget_tokens)

    @property
    def handle(self) -> ctypes.c_void_p:
        if not self._h:
            raise ValueError("tree was destroyed")
        return self._h

    def destroy(self) -> None:
        if self._h:
            _check(_lib.rt_destroy(self._h), "rt_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def rt_create(max_nodes: int, max_pool_tokens: int, budget_tokens: int = 0, vocab: int = 0, max_clock: int = 0) -> Tree:
    cfg = rt_config(int(vocab), int(max_nodes), int(max_pool_tokens), int(budget_tokens), int(max_clock))
    h = ctypes.c_void_p()
    _check(_lib.rt_create(ctypes.byref(cfg), ctypes.byref(h)), "rt_create")
    return Tree(h, budget_tokens)


def rt_build(tokens: torch.Tensor, offsets: torch.Tensor, max_nodes: int, max_pool_tokens: int,
             budget_tokens: int = 0, vocab: int = 0, max_clock: int = 0) -> Tree:
    cfg = rt_config(int(vocab), int(max_nodes), int(max_pool_tokens), int(budget_tokens), int(max_clock))
    h = ctypes.c_void_p()
    n = offsets.numel() - 1
    _check(_lib.rt_build(_dev(tokens, torch.int32, "tokens", n == 0), _dev(offsets, torch.int64, "offsets"), n,
                         ctypes.byref(cfg), _stream(), ctypes.byref(h)), "rt_build")
    return Tree(h, budget_tokens)


def rt_insert(tree: Tree, tokens: torch.Tensor, offsets: torch.Tensor, new_tokens: Optional[torch.Tensor] = None) -> None:
    n = offsets.numel() - 1
    _check(_lib.rt_insert(tree.handle, _dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"), n,
                          _dev(new_tokens, torch.int32, "new_tokens", True), _stream()), "rt_insert")


def rt_match_batch(tree: Tree, q_tokens: torch.Tensor, q_offsets: torch.Tensor, match_len: torch.Tensor,
                   term_node: Optional[torch.Tensor] = None, term_off: Optional[torch.Tensor] = None) -> None:
    nq = q_offsets.numel() - 1
    _check(_lib.rt_match_batch(tree.handle, _dev(q_tokens, torch.int32, "q_tokens"), _dev(q_offsets, torch.int64, "q_offsets"),
                               nq, _dev(match_len, torch.int32, "match_len"), _dev(term_node, torch.int32, "term_node", True),
                               _dev(term_off, torch.int32, "term_off", True), _stream()), "rt_match_batch")


def match_state_buffer(nq: int, device) -> torch.Tensor:
    """Device memory for the records rt_match_batch_ex keeps for klpm_run_ex (klpm_match_state[nq], opaque)."""
    return torch.empty((max(int(nq), 1), MATCH_STATE_BYTES // 8), dtype=torch.int64, device=device)


def rt_match_batch_ex(tree: Tree, q_tokens: torch.Tensor, q_offsets: torch.Tensor, match_len: torch.Tensor,
                      term_node: Optional[torch.Tensor] = None, term_off: Optional[torch.Tensor] = None,
                      state: Optional[torch.Tensor] = None) -> None:
    nq = q_offsets.numel() - 1
    if state is not None and state.numel() * 8 < nq * MATCH_STATE_BYTES:
        raise ValueError("state must hold %d bytes per query" % MATCH_STATE_BYTES)
    _check(_lib.rt_match_batch_ex(tree.handle, _dev(q_tokens, torch.int32, "q_tokens"), _dev(q_offsets, torch.int64, "q_offsets"),
                                  nq, _dev(match_len, torch.int32, "match_len"), _dev(term_node, torch.int32, "term_node", True),
                                  _dev(term_off, torch.int32, "term_off", True), _dev(state, torch.int64, "state", True),
                                  _stream()), "rt_match_batch_ex")


def rt_prefix_slots(tree: Tree, term_node: torch.Tensor, match_len: torch.Tensor, slots: torch.Tensor) -> None:
    """slots (int32[nq, max_len]) receives the token-pool indices of every query's match, -1 behind its end: the page
    table of the cached prefixes with pages of one token (see include/klpm.h, also for what that asks of the cache's size)."""
    nq = match_len.numel()
    if term_node.numel() != nq or slots.dim() != 2 or slots.shape[0] != nq:
        raise ValueError("term_node, match_len and the rows of slots must be one per query")
    p, stride = _table(slots, "slots")
    _check(_lib.rt_prefix_slots(tree.handle, _dev(term_node, torch.int32, "term_node"), _dev(match_len, torch.int32, "match_len"), nq,
                                p, stride, slots.shape[1], _stream()), "rt_prefix_slots")


def rt_stats(tree: Tree) -> dict:
    v = [ctypes.c_int64() for _ in range(5)]
    _check(_lib.rt_stats(tree.handle, *[ctypes.byref(x) for x in v]), "rt_stats")
    return dict(n_nodes=v[0].value, tokens=v[1].value, clock=v[2].value, evictions=v[3].value, pool_used=v[4].value)


def rt_clone(tree: Tree) -> Tree:
    h = ctypes.c_void_p()
    _check(_lib.rt_clone(tree.handle, _stream(), ctypes.byref(h)), "rt_clone")
    return Tree(h, tree.budget_tokens)


def rt_checkpoint(tree: Tree) -> None:
    _check(_lib.rt_checkpoint(tree.handle, _stream()), "rt_checkpoint")


def rt_rollback(tree: Tree) -> None:
    _check(_lib.rt_rollback(tree.handle, _stream()), "rt_rollback")


def rt_status_detail(tree: Tree) -> int:
    d = ctypes.c_int32()
    _check(_lib.rt_status_detail(tree.handle, ctypes.byref(d)), "rt_status_detail")
    return int(d.value)


def rt_sync_status(tree: Tree) -> int:
    return int(_lib.rt_sync_status(tree.handle, _stream()))


def rt_destroy(tree: Tree) -> None:
    tree.destroy()


def _same_length(match_len: torch.Tensor, arrival: torch.Tensor, waiting: torch.Tensor) -> int:
    n = match_len.numel()
    if arrival.numel() != n or waiting.numel() != n:
        raise ValueError("match_len, arrival and waiting must have the same number of elements")
    return n


def klpm_select(match_len: torch.Tensor, arrival: torch.Tensor, waiting: torch.Tensor, pick_counter: int,
                params: klpm_params, pick: torch.Tensor) -> None:
    _same_length(match_len, arrival, waiting)
    _check(_lib.klpm_select(_dev(match_len, torch.int32, "match_len"), _dev(arrival, torch.int64, "arrival"),
                            _dev(waiting, torch.uint8, "waiting"), match_len.numel(), int(pick_counter),
                            ctypes.byref(params), _dev(pick, torch.int32, "pick"), _stream()), "klpm_select")


def klpm_select_topk(match_len: torch.Tensor, arrival: torch.Tensor, waiting: torch.Tensor, out: torch.Tensor) -> None:
    """out (int32[kk]) receives the kk best longest-match candidates of this snapshot, best first."""
    _same_length(match_len, arrival, waiting)
    _check(_lib.klpm_select_topk(_dev(match_len, torch.int32, "match_len"), _dev(arrival, torch.int64, "arrival"),
                                 _dev(waiting, torch.uint8, "waiting"), match_len.numel(), out.numel(),
                                 _dev(out, torch.int32, "out"), _stream()), "klpm_select_topk")


def klpm_select_noalloc(match_len: torch.Tensor, arrival: torch.Tensor, waiting: torch.Tensor, pick_counter: int,
                        params: klpm_params, pick: torch.Tensor) -> None:
    """klpm_select without any device allocation inside the library (fixed scratch; at most
    SELECT_NOALLOC_MAX_QUERIES queries; calls must not overlap on the GPU)."""
    n = _same_length(match_len, arrival, waiting)
    _check(_lib.klpm_select_noalloc(_dev(match_len, torch.int32, "match_len"), _dev(arrival, torch.int64, "arrival"),
                                    _dev(waiting, torch.uint8, "waiting"), n, int(pick_counter),
                                    ctypes.byref(params), _dev(pick, torch.int32, "pick"), _stream()),
           "klpm_select_noalloc")


def klpm_replay(tree: Tree, order: torch.Tensor, q_tokens: torch.Tensor, q_offsets: torch.Tensor, arrival: torch.Tensor,
                params: klpm_params, uncached: torch.Tensor, ttft: torch.Tensor,
                completion: Optional[torch.Tensor] = None) -> None:
    _check(_lib.klpm_replay(tree.handle, _dev(order, torch.int32, "order"), order.numel(),
                            _dev(q_tokens, torch.int32, "q_tokens"), _dev(q_offsets, torch.int64, "q_offsets"),
                            _dev(arrival, torch.int64, "arrival"), arrival.numel(), ctypes.byref(params),
                            _dev(uncached, torch.int32, "uncached"), _dev(ttft, torch.int64, "ttft"),
                            _dev(completion, torch.int64, "completion", True), _stream()), "klpm_replay")


def klpm_run(tree: Tree, q_tokens: torch.Tensor, q_offsets: torch.Tensor, arrival: torch.Tensor, params: klpm_params,
             order: torch.Tensor, uncached: torch.Tensor, ttft: torch.Tensor,
             completion: Optional[torch.Tensor] = None) -> None:
    n = arrival.numel()
    _check(_lib.klpm_run(tree.handle, _dev(q_tokens, torch.int32, "q_tokens"), _dev(q_offsets, torch.int64, "q_offsets"),
                         _dev(arrival, torch.int64, "arrival"), n, ctypes.byref(params), _dev(order, torch.int32, "order"),
                         _dev(uncached, torch.int32, "uncached"), _dev(ttft, torch.int64, "ttft"),
                         _dev(completion, torch.int64, "completion", True), _stream()), "klpm_run")


RUN_PATH_NONE, RUN_PATH_ONE_BY_ONE, RUN_PATH_GROUPED = 0, 1, 2


def klpm_run_path(tree: Tree) -> int:
    """Which loop the last klpm_run / klpm_run_ex on this tree took (RUN_PATH_*)."""
    return int(_lib.klpm_run_path(tree.handle))


def klpm_batch_times(order: torch.Tensor, arrival: torch.Tensor, completion: torch.Tensor, batch_size: int,
                     ttft_b: torch.Tensor, completion_b: torch.Tensor, n_skipped: Optional[torch.Tensor] = None) -> None:
    n = arrival.numel()
    if completion.numel() != n or ttft_b.numel() != n or completion_b.numel() != n:
        raise ValueError("arrival, completion, ttft_b and completion_b must have one entry per query")
    _check(_lib.klpm_batch_times(_dev(order, torch.int32, "order"), order.numel(), _dev(arrival, torch.int64, "arrival"),
                                 _dev(completion, torch.int64, "completion"), n, int(batch_size),
                                 _dev(ttft_b, torch.int64, "ttft_b"), _dev(completion_b, torch.int64, "completion_b"),
                                 _dev(n_skipped, torch.int32, "n_skipped", True), _stream()), "klpm_batch_times")


LAST_ONLY_MAX_QUEUE = 1024


def klpm_run_last_only_batch(tokens: torch.Tensor, offsets: torch.Tensor, arrival: torch.Tensor,
                             tie_priority: Optional[torch.Tensor], queue_offsets: torch.Tensor, params: klpm_params,
                             order: torch.Tensor, uncached: torch.Tensor, ttft: torch.Tensor,
                             completion: Optional[torch.Tensor] = None, n_skipped: Optional[torch.Tensor] = None) -> None:
    """Many independent queues under the last-prompt cache, one warp each (see include/klpm.h)."""
    n_prompts = offsets.numel() - 1
    for t, name in ((arrival, "arrival"), (order, "order"), (uncached, "uncached"), (ttft, "ttft")):
        if t.numel() != n_prompts:
            raise ValueError("%s must have one entry per prompt" % name)
    _check(_lib.klpm_run_last_only_batch(_dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"),
                                         _dev(arrival, torch.int64, "arrival"),
                                         _dev(tie_priority, torch.int64, "tie_priority", True),
                                         _dev(queue_offsets, torch.int32, "queue_offsets"), queue_offsets.numel() - 1,
                                         ctypes.byref(params), _dev(order, torch.int32, "order"),
                                         _dev(uncached, torch.int32, "uncached"), _dev(ttft, torch.int64, "ttft"),
                                         _dev(completion, torch.int64, "completion", True),
                                         _dev(n_skipped, torch.int32, "n_skipped", True), _stream()),
           "klpm_run_last_only_batch")


def rt_debug_counters(tree: Tree) -> dict:
    """What the grouped loop of the last klpm_run on this tree did (see include/klpm.h); what a tree of that kind does not count is 0.
    cta_batch* and warp_step* are the names that agreed_*, windows and iterated_* go by in programs written before there were windows."""
    v = (_i64 * 16)()
    _check(_lib.rt_debug_counters(tree.handle, ctypes.byref(v)), "rt_debug_counters")
    names = ("careful_steps", "cta_dissolves", "fallback_scans", "fallen_back", "evictions", "cycles_tree", "cycles_scans",
             "cycles_cta_dissolves", "windows", "agreed_batches", "agreed_decisions", "iterated_batches",
             "iterated_decisions", "single_decisions", "cycles_windows", "cycles_single")
    c = dict(zip(names, [int(x) for x in v]))
    only_without = ("stretch_decisions", "lane_decisions", "most_grown", "rounds", "cycles_stretches")
    for i, name in enumerate(only_without):
        c[name] = 0 if tree.budget_tokens > 0 else int(v[2 + i])
        if tree.budget_tokens == 0:
            c[names[2 + i]] = 0
    for old, new in (("cta_batches_tried", "windows"), ("cta_batches", "agreed_batches"), ("cta_batch_decisions", "agreed_decisions"),
                     ("warp_steps", "iterated_batches"), ("warp_step_decisions", "iterated_decisions"),
                     ("cycles_cta_batches", "cycles_windows"), ("cycles_warp_steps", "cycles_single")):
        c[old] = c[new]
    return c


def klpm_debug_set(name: str, value: int) -> None:
    """Process-wide test/debug settings of the library (see include/klpm.h); value < 0 restores the default."""
    _check(_lib.klpm_debug_set(name.encode(), int(value)), "klpm_debug_set")


def klpm_run_ex(tree: Tree, q_tokens: torch.Tensor, q_offsets: torch.Tensor, arrival: torch.Tensor, params: klpm_params,
                tie_priority: Optional[torch.Tensor], score_mode: int, order: torch.Tensor, uncached: torch.Tensor,
                ttft: torch.Tensor, completion: Optional[torch.Tensor] = None,
                match_state: Optional[torch.Tensor] = None) -> None:
    n = arrival.numel()
    _check(_lib.klpm_run_ex(tree.handle, _dev(q_tokens, torch.int32, "q_tokens"), _dev(q_offsets, torch.int64, "q_offsets"),
                            _dev(arrival, torch.int64, "arrival"), n, ctypes.byref(params),
                            _dev(tie_priority, torch.int64, "tie_priority", True), int(score_mode),
                            _dev(match_state, torch.int64, "match_state", True),
                            _dev(order, torch.int32, "order"), _dev(uncached, torch.int32, "uncached"),
                            _dev(ttft, torch.int64, "ttft"), _dev(completion, torch.int64, "completion", True), _stream()),
           "klpm_run_ex")


# ---- the KV cache behind the tree (include/klpm_kv.h) ----

KV_F32, KV_BF16, KV_F16, KV_E4M3 = 0, 1, 2, 3
KV_MAX_HEAD_DIM = 256
_KV_TYPES = {torch.float32: KV_F32, torch.bfloat16: KV_BF16, torch.float16: KV_F16, torch.float8_e4m3fn: KV_E4M3}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class kv_cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("dtype", _i32), ("n_pages", _i32), ("page_size", _i32), ("n_heads", _i32),
                ("head_dim", _i32), ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float), ("k_stride", _i64 * 3),
                ("v_stride", _i64 * 3)]


class kv_rows(ctypes.Structure):
    _fields_ = [("data", _vp), ("dtype", _i32), ("n_heads", _i32), ("stride", _i64 * 2)]


class kv_rope(ctypes.Structure):
    _fields_ = [("d_turns", _vp), ("rot_dim", _i32), ("interleaved", _i32), ("factor", ctypes.c_float)]


_f32, _f64 = ctypes.c_float, ctypes.c_double
# structs are passed as addresses or as packed bytes: building a ctypes object per argument costs more than a small call's launches
_lib.kv_rope_table.restype = _i32
_lib.kv_rope_table.argtypes = [_vp, _i32, _f64, _i32, _f64, _f64, _f64, _f64, ctypes.POINTER(_f32), _vp]
_lib.kv_rope_append.restype = _i32
_lib.kv_rope_append.argtypes = [_vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp]
_lib.kv_decode_workspace.restype = _i64
_lib.kv_decode_workspace.argtypes = [_vp, _i32, _i32, _i32, _i32]
_lib.kv_decode.restype = _i32
_lib.kv_decode.argtypes = [_vp, _vp, _vp, _i32, _vp, _i64, _i32, _vp, _f32, _i32, _vp, _vp, _vp, _vp, _i64, _vp]
_lib.kv_evict.restype = _i32
_lib.kv_evict.argtypes = [_vp, _vp, _vp, _i32, _vp, _i64, _i32, _vp, _vp, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _i32, _vp, _vp]
_pack_rows, _pack_strides = struct.Struct("Pii2q").pack, struct.Struct("2q").pack      # kv_rows; int64[2]

KV_EXPORTS = ["kv_rope_table", "kv_rope_append", "kv_decode_workspace", "kv_decode", "kv_evict"]


def _stream_of(device: torch.device) -> int:
    """The current stream's handle.  The calls launch on the current device: tensors of another one are refused."""
    here = torch.cuda.current_device()
    if device.index != here:
        raise ValueError("tensors are on %s, the current device is cuda:%d" % (device, here))
    return torch._C._cuda_getCurrentRawStream(here)


class KvCache:
    """A paged KV cache: k and v are CUDA tensors [n_pages, page_size, n_heads, head_dim] (any strides, head_dim contiguous) of one
    dtype, bfloat16, float16 or float8_e4m3fn.  An 8-bit element stands for its value times k_scale (v_scale).  The tensors are kept
    alive by this object."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: float = 1.0, v_scale: float = 1.0):
        if not k.is_cuda or not v.is_cuda:
            raise ValueError("k and v must be CUDA tensors (this library has no CPU path)")
        if k.dim() != 4 or k.shape != v.shape or k.dtype is not v.dtype or k.device != v.device:
            raise ValueError("k and v must be [n_pages, page_size, n_heads, head_dim] tensors of one shape, dtype and device")
        if k.dtype not in (torch.bfloat16, torch.float16, torch.float8_e4m3fn):
            raise ValueError("a cache holds bfloat16, float16 or float8_e4m3fn")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("head_dim must be contiguous")
        self.k, self.v, self.device = k, v, k.device
        self.n_pages, self.page_size, self.n_heads, self.head_dim = k.shape
        if max(k.shape) >= 1 << 31:
            raise ValueError("a dimension of the cache is too large")
        self.c = kv_cache(k.data_ptr(), v.data_ptr(), _KV_TYPES[k.dtype], *k.shape, float(k_scale), float(v_scale),
                          (_i64 * 3)(*k.stride()[:3]), (_i64 * 3)(*v.stride()[:3]))
        self.p = ctypes.addressof(self.c)


class Rope:
    """Rotary positions as kv_rope_append takes them (made by kv_rope_table)."""

    def __init__(self, turns: torch.Tensor, rot_dim: int, interleaved: bool, factor: float):
        self.turns, self.factor = turns, factor
        self.c = kv_rope(turns.data_ptr(), rot_dim, int(interleaved), factor)
        self.p = ctypes.addressof(self.c)


def kv_rope_table(rot_dim: int, theta: float = 10_000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0,
                  original_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda") -> Rope:
    """The frequencies of rotary positions over the first rot_dim elements of a head, scaled for contexts `factor` times as long as
    original_len: scaling "none", "linear", "ntk" or "yarn" (see include/klpm_kv.h, also for checkpoints whose YaRN ramps otherwise)."""
    _count(rot_dim, "rot_dim")
    if scaling not in ROPE_SCALINGS:
        raise ValueError("scaling must be one of %s" % ", ".join(sorted(ROPE_SCALINGS)))
    turns = torch.empty(max(int(rot_dim) // 2, 1), dtype=torch.float64, device=device)
    stream = _stream_of(turns.device)
    f = _f32()
    _check(_lib.kv_rope_table(turns.data_ptr(), int(rot_dim), float(theta), ROPE_SCALINGS[scaling], float(factor), float(original_len),
                              float(beta_fast), float(beta_slow), ctypes.byref(f), stream), "kv_rope_table")
    return Rope(turns, int(rot_dim), interleaved, f.value)


def _rows(t: torch.Tensor, cache: KvCache, n: int, name: str) -> bytes:
    shape, stride, dtype = t.shape, t.stride(), _KV_TYPES.get(t.dtype)
    if len(shape) != 3 or shape[0] != n or shape[2] != cache.head_dim or (stride[2] != 1 and shape[2] > 1):
        raise ValueError("%s must be [%d, heads, %d] with contiguous head_dim" % (name, n, cache.head_dim))
    if dtype is None or t.device != cache.device:
        raise ValueError("%s must be a floating-point tensor on the cache's device" % name)
    return _pack_rows(t.data_ptr(), dtype, shape[1], stride[0], stride[1])


def _ints(t: torch.Tensor, cache: KvCache, n: int, name: str) -> int:
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of %d elements" % (name, n))
    if t.device != cache.device:
        raise ValueError("%s must be on the cache's device" % name)
    return t.data_ptr()


def _pages(t: torch.Tensor, cache: KvCache, n: int, name: str):
    """Pointer, row stride and width of a page table."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not torch.int32 or len(shape) != 2 or shape[0] != n or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("%s must be an int32 tensor with one contiguous row per sequence" % name)
    if t.device != cache.device:
        raise ValueError("%s must be on the cache's device" % name)
    return t.data_ptr(), stride[0], shape[1]


def _count(x: int, name: str) -> int:
    """A number that fits the C call's int32."""
    if not 0 <= x < 1 << 31:
        raise ValueError("%s must be between 0 and 2^31 - 1" % name)
    return x


def kv_rope_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
                   rope: Optional[Rope] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> None:
    """Rotate q [n, q_heads, head_dim] into q_out and k by positions (int32[n]), and store k and v [n, n_heads, head_dim] at slots
    (int32[n]) of the cache.  q_out may be q.  Without rope nothing is rotated; rows with a slot out of range are not stored."""
    n = slots.numel()
    at = p = None
    if rope is not None:
        if positions is None:
            raise ValueError("rope needs one position per row")
        if rope.turns.device != cache.device:
            raise ValueError("the table of rope must be on the cache's device")
        p = rope.p
    if positions is not None:
        at = _ints(positions, cache, n, "positions")
    rq = ro = None
    if q is not None and q_out is not None:
        rq = _rows(q, cache, n, "q")
        ro = rq if q_out is q else _rows(q_out, cache, n, "q_out")
    elif q is not None or q_out is not None:
        raise ValueError("q and q_out go together")
    _check(_lib.kv_rope_append(cache.p, p, at, _ints(slots, cache, n, "slots"), n, rq, ro, _rows(k, cache, n, "k"), _rows(v, cache, n, "v"),
                               _stream_of(cache.device)), "kv_rope_append")


def kv_decode_workspace(cache: KvCache, n_seqs: int, n_q_heads: int, max_pages: int, with_weight: bool = False) -> torch.Tensor:
    """Device memory for the workspace of a kv_decode of these sizes.  One call uses it at a time."""
    n = _lib.kv_decode_workspace(cache.p, _count(n_seqs, "n_seqs"), _count(n_q_heads, "n_q_heads"), _count(max_pages, "max_pages"), int(with_weight))
    if n < 0:
        _check(n, "kv_decode_workspace")
    return torch.empty(max(n, 256), dtype=torch.uint8, device=cache.device)


def _weight(t: torch.Tensor, cache: KvCache, n: int, least: int, name: str):
    shape, stride = t.shape, t.stride()
    if t.dtype is not torch.float32 or len(shape) != 3 or shape[0] != n or shape[1] != cache.n_heads or shape[2] < least \
            or (stride[2] != 1 and shape[2] > 1):
        raise ValueError("%s must be a float32 [%d, %d, >= %d] tensor with contiguous rows" % (name, n, cache.n_heads, least))
    if t.device != cache.device:
        raise ValueError("%s must be on the cache's device" % name)
    return t.data_ptr(), _pack_strides(stride[0], stride[1])


def kv_decode(cache: KvCache, q: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, out: torch.Tensor,
              scale: Optional[float] = None, window: int = 0, lse: Optional[torch.Tensor] = None,
              weight: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Attention of one new token per sequence: q, out [n_seqs, q_heads, head_dim], page_table int32[n_seqs, max_pages], lengths
    int32[n_seqs].  scale defaults to head_dim ** -0.5.  lse float32[n_seqs, q_heads] receives the logarithm of the softmax's sum;
    weight float32[n_seqs, n_heads, max_pages * page_size] is increased by what every cached token received.  Without a
    workspace (kv_decode_workspace) the call takes one from torch's allocator; with weight that is 4 bytes per sequence, query head and token of the
    table's width, whatever the lengths are."""
    n = lengths.numel()
    table, stride, max_pages = _pages(page_table, cache, n, "page_table")
    rq = _rows(q, cache, n, "q")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.device != cache.device):
        raise ValueError("lse must be a contiguous float32 [n_seqs, q_heads] tensor on the cache's device")
    w, ws = _weight(weight, cache, n, max_pages * cache.page_size, "weight") if weight is not None else (None, None)
    if workspace is None:
        workspace = kv_decode_workspace(cache, n, q.shape[1], max_pages, weight is not None)
    elif workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.device != cache.device:
        raise ValueError("workspace must be a contiguous uint8 tensor on the cache's device")
    _check(_lib.kv_decode(cache.p, rq, _rows(out, cache, n, "out"), n, table, stride, max_pages, _ints(lengths, cache, n, "lengths"),
                          cache.head_dim ** -0.5 if scale is None else scale, _count(window, "window"), lse.data_ptr() if lse is not None else None, w, ws,
                          workspace.data_ptr(), workspace.numel(), _stream_of(cache.device)), "kv_decode")


def kv_evict(cache: KvCache, weight: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, new_table: torch.Tensor, keep: int,
             sinks: int = 0, recent: int = 0, *, index: torch.Tensor, new_weight: torch.Tensor, new_lengths: torch.Tensor) -> None:
    """Shorten every sequence to `keep` tokens per cache head: the first `sinks`, the last `recent`, then the largest weight
    (float32[n_seqs, n_heads, >= max_pages * page_size]).  They are copied to the pages of new_table (int32[n_seqs, new_pages]), which
    must not be pages of page_table; index int32[n_seqs, n_heads, keep], new_weight float32[n_seqs, n_heads, >= keep] and new_lengths
    int32[n_seqs] receive which, their weights, and how many."""
    n = lengths.numel()
    table, stride, max_pages = _pages(page_table, cache, n, "page_table")
    fresh, fresh_stride, new_pages = _pages(new_table, cache, n, "new_table")
    if tuple(index.shape) != (n, cache.n_heads, keep):
        raise ValueError("index must be [n_seqs, n_heads, keep]")
    w, ws = _weight(weight, cache, n, max_pages * cache.page_size, "weight")
    nw, nws = _weight(new_weight, cache, n, keep, "new_weight")
    _check(_lib.kv_evict(cache.p, w, ws, n, table, stride, max_pages, _ints(lengths, cache, n, "lengths"), fresh, fresh_stride, new_pages, _count(keep, "keep"),
                         _count(sinks, "sinks"), _count(recent, "recent"), _ints(index, cache, n * cache.n_heads * keep, "index"), nw, nws, new_weight.shape[2],
                         _ints(new_lengths, cache, n, "new_lengths"), _stream_of(cache.device)), "kv_evict")
