"""Python binding of ``libbf.so`` (C ABI in ``include/bf.h``).

Argument marshalling only: every step of the search runs in the library's
CUDA kernels.  PyTorch supplies device buffers (``eval_mappings`` outputs) and
streams (``torch.cuda.current_stream()`` by default).  The functions mirror
the C entry points without their ``bf_`` prefix: ``validate_desc``,
``create_scenario``, ``destroy_scenario``, ``eval_mappings``, ``search_best``,
``search_range``, ``search_batch``, ``search_batch_noalloc``, ``eval_indices``,
``whatif``, ``search_pruned``, ``set_wait_timeout_ms``, ``last_error``,
``version``; and, for learning from the makespans of sampled mappings,
``token_logprobs``, ``token_logprobs_grad``, ``policy_loss``,
``preference_loss``, ``embed`` and ``embed_grad``; and, for a decoding step of
the model that samples them, ``prefix_attention``, ``beam_step`` and
``beam_reorder``.  Those nine are outside autograd: what they return has no graph, also where an argument requires a
gradient.  A loss's ``grad`` is the gradient in the logits, to hand to torch
(``logits.backward(loss.grad)``); an ``out`` is marked as written over.

There is no CPU fallback: if ``libbf.so`` has not been built, or no CUDA
device is present, these calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes
import dataclasses
import functools
import itertools
import os
from typing import List, NamedTuple, Optional, Sequence, Tuple, Union

from .scenarios import MAX_TOOLS, Scenario

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_build", "libbf.so")

BF_OK, BF_EINVAL, BF_ERANGE, BF_ENOMEM, BF_ECUDA, BF_ETIMEOUT = range(6)
STATUS_NAMES = {0: "BF_OK", 1: "BF_EINVAL", 2: "BF_ERANGE", 3: "BF_ENOMEM", 4: "BF_ECUDA", 5: "BF_ETIMEOUT"}
INFEASIBLE = 0xFFFFFFFF
EXPORTED = ("bf_validate_desc", "bf_create_scenario", "bf_destroy_scenario", "bf_eval_mappings",
            "bf_search_best", "bf_search_range", "bf_search_batch", "bf_search_batch_noalloc",
            "bf_eval_indices", "bf_whatif", "bf_search_pruned", "bf_search_tree", "bf_token_logprobs",
            "bf_token_logprobs_grad", "bf_policy_loss", "bf_policy_loss_workspace", "bf_preference_loss",
            "bf_preference_loss_workspace", "bf_embed", "bf_embed_grad", "bf_embed_grad_workspace",
            "bf_prefix_attention", "bf_prefix_attention_workspace", "bf_beam_step", "bf_beam_step_workspace",
            "bf_beam_reorder", "bf_set_wait_timeout_ms", "bf_last_error", "bf_version")
SPACE_BINARY, SPACE_FULL = 2, 3
TREE_NO_PRUNE = 1
MAX_PROBES = 2 * MAX_TOOLS + MAX_TOOLS * MAX_TOOLS
NOALLOC_MAX_SCENARIOS = 1024


class BfError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {message}")
        self.code = code
        self.message = message


U32xT = ctypes.c_uint32 * MAX_TOOLS


class Desc(ctypes.Structure):
    """``bf_scenario_desc``."""
    _fields_ = [("n", ctypes.c_uint32), ("pred_mask", U32xT), ("cpu_us", U32xT), ("gpu_us", U32xT),
                ("xfer_us", U32xT), ("load_us", U32xT), ("vram_mib", U32xT),
                ("vram_budget_mib", ctypes.c_uint32), ("slowdown_q10", ctypes.c_uint32 * (MAX_TOOLS + 1))]


class CResult(ctypes.Structure):
    """``bf_result``."""
    _fields_ = [("index", ctypes.c_uint64), ("makespan_us", ctypes.c_uint32), ("feasible", ctypes.c_uint32),
                ("mode", ctypes.c_uint8 * MAX_TOOLS)]


class CProbe(ctypes.Structure):
    """``bf_probe``."""
    _fields_ = [("index", ctypes.c_uint64), ("makespan_us", ctypes.c_uint32), ("feasible", ctypes.c_uint32),
                ("kind", ctypes.c_uint8), ("tool", ctypes.c_uint8), ("mode", ctypes.c_uint8),
                ("other", ctypes.c_uint8)]


@dataclasses.dataclass
class Probe:
    """One what-if probe of Algorithm 1: kind 'single' (tool -> mode) or 'swap'
    (tool -> gpu_now, other -> gpu_queue)."""
    kind: str
    tool: int
    mode: int
    other: Optional[int]
    index: int
    makespan_us: int
    feasible: bool


class CTreeStats(ctypes.Structure):
    """``bf_tree_stats``."""
    _fields_ = [("nodes", ctypes.c_uint64), ("leaf_nodes", ctypes.c_uint64), ("leaves", ctypes.c_uint64),
                ("launches", ctypes.c_uint32), ("leaf_depth", ctypes.c_uint32), ("incumbent_us", ctypes.c_uint32),
                ("pad", ctypes.c_uint32)]


class Matrix(ctypes.Structure):
    """``bf_matrix``."""
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64),
                ("row_stride", ctypes.c_uint64), ("dtype", ctypes.c_uint32), ("pad", ctypes.c_uint32)]


class PolicyArgs(ctypes.Structure):
    """``bf_policy_args``."""
    _fields_ = [("tokens", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("old_logprob", ctypes.c_void_p),
                ("ref_logprob", ctypes.c_void_p), ("advantage", ctypes.c_void_p), ("sequences", ctypes.c_uint64),
                ("advantage_per_token", ctypes.c_uint32), ("reduction", ctypes.c_uint32),
                ("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float), ("kl_coef", ctypes.c_float),
                ("entropy_coef", ctypes.c_float), ("temperature", ctypes.c_float), ("grad_scale", ctypes.c_float)]


class PreferenceArgs(ctypes.Structure):
    """``bf_preference_args``."""
    _fields_ = [("tokens", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("ref_logprob", ctypes.c_void_p),
                ("pairs", ctypes.c_uint64), ("average", ctypes.c_uint32), ("beta", ctypes.c_float),
                ("label_smoothing", ctypes.c_float), ("margin", ctypes.c_float), ("temperature", ctypes.c_float),
                ("grad_scale", ctypes.c_float)]


class Cache(ctypes.Structure):
    """``bf_cache``."""
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_uint64), ("tokens", ctypes.c_uint64),
                ("heads", ctypes.c_uint64), ("dim", ctypes.c_uint64), ("batch_stride", ctypes.c_uint64),
                ("token_stride", ctypes.c_uint64), ("head_stride", ctypes.c_uint64), ("dtype", ctypes.c_uint32),
                ("pad", ctypes.c_uint32)]


class AttentionArgs(ctypes.Structure):
    """``bf_attention_args``."""
    _fields_ = [("prefix_lengths", ctypes.c_void_p), ("suffix_lengths", ctypes.c_void_p), ("scale", ctypes.c_float),
                ("pad", ctypes.c_uint32)]


class BeamArgs(ctypes.Structure):
    """``bf_beam_args``."""
    _fields_ = [("scores", ctypes.c_void_p), ("finished", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("groups", ctypes.c_uint64), ("beams", ctypes.c_uint32), ("keep", ctypes.c_uint32),
                ("end_token", ctypes.c_int64), ("length_penalty", ctypes.c_float), ("temperature", ctypes.c_float)]


class States(ctypes.Structure):
    """``bf_states``."""
    _fields_ = [("rows", ctypes.c_uint64), ("tokens", ctypes.c_uint64), ("heads", ctypes.c_uint64),
                ("width", ctypes.c_uint64), ("row_stride", ctypes.c_uint64), ("token_stride", ctypes.c_uint64),
                ("head_stride", ctypes.c_uint64)]


@dataclasses.dataclass
class Result:
    index: int
    makespan_us: int
    feasible: bool
    modes: List[int]


_lib = None


def load(path: str = LIB_PATH):
    """Load libbf.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(path)
    vp, u64, u32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32
    lib.bf_validate_desc.argtypes = [ctypes.POINTER(Desc)]
    lib.bf_create_scenario.argtypes = [ctypes.POINTER(Desc), ctypes.POINTER(vp)]
    lib.bf_destroy_scenario.argtypes = [vp]
    lib.bf_eval_mappings.argtypes = [vp, u64, u64, vp, vp, vp]
    lib.bf_search_best.argtypes = [vp, ctypes.POINTER(CResult), vp]
    lib.bf_search_range.argtypes = [vp, u64, u64, ctypes.POINTER(CResult), vp]
    lib.bf_search_batch.argtypes = [ctypes.POINTER(Desc), u32, ctypes.POINTER(CResult), vp]
    lib.bf_search_batch_noalloc.argtypes = [ctypes.POINTER(Desc), u32, ctypes.POINTER(CResult), vp]
    lib.bf_eval_indices.argtypes = [vp, vp, u64, vp, vp, vp]
    lib.bf_whatif.argtypes = [vp, u64, ctypes.POINTER(CProbe), u32, ctypes.POINTER(u32), vp]
    lib.bf_search_pruned.argtypes = [vp, u64, ctypes.POINTER(CResult), vp]
    lib.bf_search_tree.argtypes = [vp, u32, u32, u64, ctypes.POINTER(CResult), ctypes.POINTER(CTreeStats), vp]
    mat, f32 = ctypes.POINTER(Matrix), ctypes.c_float
    lib.bf_token_logprobs.argtypes = [mat, vp, f32, vp, vp, vp]
    lib.bf_token_logprobs_grad.argtypes = [mat, vp, f32, vp, vp, mat, vp]
    lib.bf_policy_loss.argtypes = [mat, ctypes.POINTER(PolicyArgs), vp, vp, mat, vp, u64, vp]
    lib.bf_preference_loss.argtypes = [mat, ctypes.POINTER(PreferenceArgs), vp, vp, vp, mat, vp, u64, vp]
    lib.bf_embed.argtypes = [mat, vp, f32, mat, vp]
    lib.bf_embed_grad.argtypes = [mat, vp, f32, u32, mat, vp, u64, vp]
    states, table = ctypes.POINTER(States), ctypes.POINTER(vp)
    lib.bf_prefix_attention.argtypes = [vp] * 9 + [u64, vp]  # bf_cache, bf_attention_args by address: prefix_attention
    lib.bf_prefix_attention_workspace.argtypes = [vp, vp, vp, ctypes.POINTER(u64)]
    lib.bf_beam_step.argtypes = [vp] * 8 + [u64, vp]  # bf_matrix, bf_beam_args by address: beam_step
    lib.bf_beam_step_workspace.argtypes = [u64, u32, u64, u32, ctypes.POINTER(u64)]
    lib.bf_beam_reorder.argtypes = [table, states, table, states, u32, vp, u32, vp, vp]
    for name in ("bf_policy_loss_workspace", "bf_preference_loss_workspace", "bf_embed_grad_workspace"):
        getattr(lib, name).argtypes = [u64, u64, ctypes.POINTER(u64)]
    for name in EXPORTED:
        getattr(lib, name).restype = ctypes.c_int
    lib.bf_set_wait_timeout_ms.argtypes = [u32]
    lib.bf_set_wait_timeout_ms.restype = None
    lib.bf_last_error.restype = ctypes.c_char_p
    lib.bf_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(code: int):
    if code != BF_OK:
        raise BfError(code, last_error())


def last_error() -> str:
    return load().bf_last_error().decode()


def version() -> str:
    return load().bf_version().decode()


def set_wait_timeout_ms(ms: int) -> None:
    load().bf_set_wait_timeout_ms(ms)


def to_desc(scn: Scenario) -> Desc:
    d = Desc()
    d.n = scn.n
    for name in ("pred_mask", "cpu_us", "gpu_us", "xfer_us", "load_us", "vram_mib"):
        arr = getattr(d, name)
        for i, v in enumerate(getattr(scn, name)[:MAX_TOOLS]):
            arr[i] = v
    d.vram_budget_mib = scn.vram_budget_mib
    for k, v in enumerate(scn.slowdown_q10[:MAX_TOOLS + 1]):
        d.slowdown_q10[k] = v
    return d


DESC_WORDS = ctypes.sizeof(Desc) // 4


def pack_descs(scns: Sequence[Scenario]):
    """Pack scenarios into a contiguous (count, DESC_WORDS) uint32 array laid out as bf_scenario_desc[]."""
    import numpy as np
    count = len(scns)
    arr = np.zeros((count, DESC_WORDS), dtype=np.uint32)
    if count == 0:
        return arr
    cols = ("pred_mask", "cpu_us", "gpu_us", "xfer_us", "load_us", "vram_mib")
    sizes = {sc.n for sc in scns}
    if len(sizes) == 1:  # one tool count: fill whole columns at once
        n = sizes.pop()
        arr[:, 0] = n
        flat = lambda rows, width: np.fromiter(itertools.chain.from_iterable(rows), dtype=np.uint32,
                                               count=count * width).reshape(count, width)
        for j, name in enumerate(cols):
            arr[:, 1 + MAX_TOOLS * j: 1 + MAX_TOOLS * j + n] = flat((getattr(sc, name)[:n] for sc in scns), n)
        arr[:, 1 + 6 * MAX_TOOLS] = np.fromiter((sc.vram_budget_mib for sc in scns), dtype=np.uint32, count=count)
        pad = [0] * (MAX_TOOLS + 1)
        arr[:, 2 + 6 * MAX_TOOLS:] = flat(((sc.slowdown_q10 + pad)[:MAX_TOOLS + 1] for sc in scns), MAX_TOOLS + 1)
        return arr
    for r, sc in enumerate(scns):
        arr[r, 0] = sc.n
        for j, name in enumerate(cols):
            arr[r, 1 + MAX_TOOLS * j: 1 + MAX_TOOLS * j + sc.n] = getattr(sc, name)[:sc.n]
        arr[r, 1 + 6 * MAX_TOOLS] = sc.vram_budget_mib
        f = sc.slowdown_q10[:MAX_TOOLS + 1]
        arr[r, 2 + 6 * MAX_TOOLS: 2 + 6 * MAX_TOOLS + len(f)] = f
    return arr


def _result(r: CResult, n: int) -> Result:
    return Result(int(r.index), int(r.makespan_us), bool(r.feasible), [int(r.mode[i]) for i in range(n)])


def _stream_handle(stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def validate_desc(scn: Scenario) -> None:
    """Raise BfError(BF_EINVAL) if the scenario is outside the library's limits."""
    d = to_desc(scn)
    _check(load().bf_validate_desc(ctypes.byref(d)))


class ScenarioHandle:
    """An owned ``bf_scenario*``; released by :meth:`close` (or garbage collection)."""

    def __init__(self, scn: Scenario):
        self.scenario = scn
        self._ptr = ctypes.c_void_p()
        d = to_desc(scn)
        _check(load().bf_create_scenario(ctypes.byref(d), ctypes.byref(self._ptr)))

    @property
    def ptr(self):
        if not self._ptr:
            raise ValueError("scenario handle is closed")
        return self._ptr

    def close(self):
        if self._ptr:
            ptr, self._ptr = self._ptr, ctypes.c_void_p()
            _check(load().bf_destroy_scenario(ptr))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def create_scenario(scn: Scenario) -> ScenarioHandle:
    return ScenarioHandle(scn)


def destroy_scenario(handle: ScenarioHandle) -> None:
    handle.close()


def _handle(h: Union[ScenarioHandle, Scenario]) -> Tuple[ScenarioHandle, bool]:
    if isinstance(h, ScenarioHandle):
        return h, False
    return ScenarioHandle(h), True


def _check_out(out_makespan, out_feasible, count: int) -> None:
    """Output buffers: contiguous CUDA tensors of >= count 4-byte / 1-byte elements."""
    for t, size, name in ((out_makespan, 4, "out_makespan"), (out_feasible, 1, "out_feasible")):
        if not (t.is_cuda and t.is_contiguous() and t.element_size() == size and t.numel() >= count):
            raise ValueError(f"{name} must be a contiguous CUDA tensor of >= {count} {size}-byte elements")


def eval_mappings(h: Union[ScenarioHandle, Scenario], first: int, count: int, out_makespan=None,
                  out_feasible=None, stream=None):
    """Makespans (torch.int32 CUDA tensor holding u32 bit patterns) and feasibility
    flags (torch.uint8) of mappings [first, first+count).  Asynchronous on ``stream``;
    the scenario's tables travel by value with the launch, and the memory of a
    handle's segment tables is freed after the work that reads it, so a temporary
    handle may be released as soon as the call returns."""
    import torch
    handle, owned = _handle(h)
    try:
        if out_makespan is None:
            out_makespan = torch.empty(count, dtype=torch.int32, device="cuda")
        if out_feasible is None:
            out_feasible = torch.empty(count, dtype=torch.uint8, device="cuda")
        _check_out(out_makespan, out_feasible, count)
        _check(load().bf_eval_mappings(handle.ptr, first, count, ctypes.c_void_p(out_makespan.data_ptr()),
                                       ctypes.c_void_p(out_feasible.data_ptr()),
                                       ctypes.c_void_p(_stream_handle(stream))))
        return out_makespan, out_feasible
    finally:
        if owned:
            handle.close()


def search_best(h: Union[ScenarioHandle, Scenario], stream=None) -> Result:
    """Optimal feasible mapping over all 3^n (ties to the lowest index)."""
    handle, owned = _handle(h)
    try:
        r = CResult()
        _check(load().bf_search_best(handle.ptr, ctypes.byref(r), ctypes.c_void_p(_stream_handle(stream))))
        return _result(r, handle.scenario.n)
    finally:
        if owned:
            handle.close()


def search_range(h: Union[ScenarioHandle, Scenario], first: int, count: int, stream=None) -> Result:
    """Best feasible mapping in [first, first+count) (feasible=False if none)."""
    handle, owned = _handle(h)
    try:
        r = CResult()
        _check(load().bf_search_range(handle.ptr, first, count, ctypes.byref(r),
                                      ctypes.c_void_p(_stream_handle(stream))))
        return _result(r, handle.scenario.n)
    finally:
        if owned:
            handle.close()


def _batch_call(fn, scns: Sequence[Scenario], stream, packed=None) -> List[Result]:
    count = len(scns)
    if packed is None and count:
        packed = pack_descs(scns)
    descs = packed.ctypes.data_as(ctypes.POINTER(Desc)) if count else None
    results = (CResult * max(count, 1))()
    _check(fn(descs, count, results, ctypes.c_void_p(_stream_handle(stream))))
    if not count:
        return []
    import numpy as np
    arr = np.ctypeslib.as_array(results)  # one structured view instead of per-field ctypes reads
    width = max(sc.n for sc in scns)
    modes = arr["mode"][:, :width].tolist()
    # Rows of full width are taken as they are: a copy of each is one more object per result for the collector.
    return [Result(i, m, bool(f), md if sc.n == width else md[:sc.n]) for i, m, f, md, sc in
            zip(arr["index"].tolist(), arr["makespan_us"].tolist(), arr["feasible"].tolist(), modes, scns)]


def search_batch(scns: Sequence[Scenario], stream=None, packed=None) -> List[Result]:
    """Full search of each scenario, the whole batch in one call.  ``packed`` (from
    :func:`pack_descs` of the same scenarios) skips the packing when a batch is searched repeatedly."""
    return _batch_call(load().bf_search_batch, scns, stream, packed)


def search_batch_noalloc(scns: Sequence[Scenario], stream=None) -> List[Result]:
    """As :func:`search_batch`, but the library allocates no memory for the call.

    For callers that cannot allocate device memory while they search (their GPU
    memory belongs to another allocator's pool, or a cudaMalloc/cudaFree pair
    would synchronise the device inside a latency-critical loop).  The scratch is
    a fixed array in the library's device image; at most NOALLOC_MAX_SCENARIOS
    scenarios per call.  Calls on one device are serialised; after a call that
    timed out, the next one first waits for that call's stream.
    """
    return _batch_call(load().bf_search_batch_noalloc, scns, stream)


def eval_indices(h: Union[ScenarioHandle, Scenario], indices, out_makespan=None, out_feasible=None, stream=None):
    """Makespans (torch.int32, u32 bit patterns) and flags (torch.uint8; 0xFF for an
    index outside [0, 3^n)) of the mappings in `indices` (a CUDA int64 tensor)."""
    import torch
    if not (indices.is_cuda and indices.dtype == torch.int64 and indices.is_contiguous()):
        raise ValueError("indices must be a contiguous CUDA int64 tensor")
    handle, owned = _handle(h)
    try:
        count = indices.numel()
        if out_makespan is None:
            out_makespan = torch.empty(count, dtype=torch.int32, device=indices.device)
        if out_feasible is None:
            out_feasible = torch.empty(count, dtype=torch.uint8, device=indices.device)
        _check_out(out_makespan, out_feasible, count)
        _check(load().bf_eval_indices(handle.ptr, ctypes.c_void_p(indices.data_ptr()), count,
                                      ctypes.c_void_p(out_makespan.data_ptr()),
                                      ctypes.c_void_p(out_feasible.data_ptr()),
                                      ctypes.c_void_p(_stream_handle(stream))))
        return out_makespan, out_feasible
    finally:
        if owned:
            handle.close()


def whatif(h: Union[ScenarioHandle, Scenario], base_index: int, stream=None) -> List[Probe]:
    """The single-tool and swap reprobes of Algorithm 1 around `base_index`, scored on the GPU."""
    handle, owned = _handle(h)
    try:
        out = (CProbe * MAX_PROBES)()
        count = ctypes.c_uint32(0)
        _check(load().bf_whatif(handle.ptr, base_index, out, MAX_PROBES, ctypes.byref(count),
                                ctypes.c_void_p(_stream_handle(stream))))
        return [Probe("swap" if p.kind else "single", p.tool, p.mode, None if p.kind == 0 else p.other,
                      p.index, p.makespan_us, bool(p.feasible)) for p in out[:count.value]]
    finally:
        if owned:
            handle.close()


def search_pruned(h: Union[ScenarioHandle, Scenario], hint_index: Optional[int] = None, stream=None) -> Result:
    """The optimum of :func:`search_best`, found by branch and bound (exact)."""
    handle, owned = _handle(h)
    try:
        r = CResult()
        hint = (1 << 64) - 1 if hint_index is None else hint_index
        _check(load().bf_search_pruned(handle.ptr, hint, ctypes.byref(r), ctypes.c_void_p(_stream_handle(stream))))
        return _result(r, handle.scenario.n)
    finally:
        if owned:
            handle.close()


def search_tree(h: Union[ScenarioHandle, Scenario], space: int = SPACE_FULL, prune: bool = True,
                hint_index: Optional[int] = None, stream=None) -> Tuple[Result, dict]:
    """Optimum of the full (space=3) or binary cpu/gpu_now (space=2) decision space of a scenario of up to
    32 tools, by depth-first branch and bound (prune=False: every mapping simulated); (result, stats)."""
    handle, owned = _handle(h)
    try:
        r = CResult()
        st = CTreeStats()
        hint = (1 << 64) - 1 if hint_index is None else hint_index
        _check(load().bf_search_tree(handle.ptr, space, 0 if prune else TREE_NO_PRUNE, hint, ctypes.byref(r),
                                     ctypes.byref(st), ctypes.c_void_p(_stream_handle(stream))))
        stats = dict(nodes=st.nodes, leaf_nodes=st.leaf_nodes, leaves=st.leaves, launches=st.launches,
                     leaf_depth=st.leaf_depth, incumbent_us=st.incumbent_us)
        return _result(r, handle.scenario.n), stats
    finally:
        if owned:
            handle.close()


# ---- learning from makespans ----------------------------------------------------------------------------------------

REDUCTIONS = {"tokens": 0, "sequences": 1, "sum": 2}
POLICY_STATS, PREFERENCE_STATS = 6, 4


class PolicyLoss(NamedTuple):
    """``stats`` (POLICY_STATS float32: loss, surrogate term, KL, entropy, clipped share, mean ratio), the tokens'
    log-probabilities and the gradient in the logits (None when not wanted)."""
    stats: object
    logprob: object
    grad: object


class PreferenceLoss(NamedTuple):
    """``stats`` (PREFERENCE_STATS float32: loss, share of pairs ranked right, mean reward of the preferred and of the
    other answers), the answers' rewards, the tokens' log-probabilities and the gradient in the logits (or None)."""
    stats: object
    rewards: object
    logprob: object
    grad: object


_DTYPE_CODES = {}


def _dtype_code(dtype) -> Optional[int]:
    if not _DTYPE_CODES:
        import torch
        _DTYPE_CODES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    return _DTYPE_CODES.get(dtype)


def _matrix(t, name: str) -> Matrix:
    """A 2-D CUDA tensor with contiguous rows (any row stride) on the current device as ``bf_matrix``."""
    import torch
    code = _dtype_code(t.dtype)
    if code is None or not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D CUDA tensor of float32, bfloat16 or float16")
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on device {t.get_device()} but device {torch.cuda.current_device()} is current")
    rows, cols = t.shape
    stride, inner = t.stride()
    if inner != 1 and cols > 1 and rows:
        raise ValueError(f"{name} must have contiguous rows")
    return Matrix(t.data_ptr(), rows, cols, max(stride, cols) if rows <= 1 else stride, code, 0)


def _vector(t, count: int, dtype, like, name: str) -> int:
    """The address of a contiguous 1-D CUDA tensor of `count` elements beside `like`."""
    if t.dtype != dtype or t.numel() != count or t.get_device() != like.get_device() or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {count} elements on {like.device}")
    return t.data_ptr()


_SAME = contextlib.nullcontext()


def _allocate(stream):
    """Context in which results and workspaces belong to `stream` for torch's allocator."""
    if stream is None:
        return _SAME
    import torch
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


def _stream_of(stream, like) -> int:
    """As _stream_handle, without the object that torch.cuda.current_stream makes (3 us of a call of 20)."""
    if stream is not None:
        return _stream_handle(stream)
    import torch
    return torch._C._cuda_getCurrentRawStream(like.get_device())


@functools.lru_cache(maxsize=256)
def _workspace_bytes(name: str, rows: int, groups: int) -> int:
    need = ctypes.c_uint64(0)
    _check(getattr(load(), name)(rows, groups, ctypes.byref(need)))
    return max(need.value, 1)


def _workspace(name: str, rows: int, groups: int, device):
    import torch
    return torch.empty(_workspace_bytes(name, rows, groups), dtype=torch.uint8, device=device)


def _written(t) -> None:
    """Tell autograd that a call wrote over a caller's tensor, as torch's own in-place operations do: it then refuses a
    backward pass that needs what the tensor held."""
    import torch
    if t is not None and not t.is_inference():
        torch.autograd.graph.increment_version(t)


def _grad_like(logits, out, grad: bool):
    """Where the gradient goes: nowhere, to `out` (it may be `logits`) or to a new tensor."""
    import torch
    if not grad:
        return None
    return torch.empty_like(logits, memory_format=torch.contiguous_format) if out is None else out


def token_logprobs(logits, tokens, *, temperature: float = 1.0, entropy: bool = False, stream=None):
    """Log-probabilities (float32) of `tokens` (int64, one per row; below 0: not scored) under `logits`
    (rows x vocab; float32, bfloat16 or float16) -- with ``entropy``, the pair of them and the rows' entropies.
    Asynchronous on ``stream``, as everything below."""
    import torch
    x = _matrix(logits, "logits")
    y = _vector(tokens, x.rows, torch.int64, logits, "tokens")
    with _allocate(stream):
        logprob = torch.empty(x.rows, dtype=torch.float32, device=logits.device)
        h = torch.empty_like(logprob) if entropy else None
    _check(load().bf_token_logprobs(x, y, temperature, logprob.data_ptr(), h.data_ptr() if entropy else None,
                                    _stream_of(stream, logits)))
    return (logprob, h) if entropy else logprob


def token_logprobs_grad(logits, tokens, grad_logprob, grad_entropy=None, *, temperature: float = 1.0, out=None,
                        stream=None):
    """The gradient in `logits` of sum(grad_logprob * logprob + grad_entropy * entropy).  `out` may be `logits`."""
    import torch
    x = _matrix(logits, "logits")
    y = _vector(tokens, x.rows, torch.int64, logits, "tokens")
    gl = _vector(grad_logprob, x.rows, torch.float32, logits, "grad_logprob")
    gh = None if grad_entropy is None else _vector(grad_entropy, x.rows, torch.float32, logits, "grad_entropy")
    with _allocate(stream):
        grad = _grad_like(logits, out, True)
    _check(load().bf_token_logprobs_grad(x, y, temperature, gl, gh, _matrix(grad, "out"), _stream_of(stream, logits)))
    _written(out)
    return grad


def policy_loss(logits, tokens, offsets, old_logprob, advantage, ref_logprob=None, *, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, temperature: float = 1.0,
                reduction: str = "tokens", advantage_per_token: bool = False, grad_scale: float = 1.0,
                grad: bool = True, out=None, stream=None) -> PolicyLoss:
    """The clipped policy loss with a KL term over the sequences that `offsets` (int64, sequences + 1) cuts the rows
    into, and its gradient in the logits (times `grad_scale`).  `advantage` holds one value per sequence, or one per row
    with `advantage_per_token`.  ``reduction``: "tokens", "sequences" or "sum".  `out` may be `logits`: the gradient
    then replaces them."""
    import torch
    x = _matrix(logits, "logits")
    rows, sequences = x.rows, offsets.numel() - 1
    if sequences < 0:
        raise ValueError("offsets must hold one element more than there are sequences")
    if reduction not in REDUCTIONS:
        raise ValueError(f"reduction must be one of {', '.join(REDUCTIONS)}")
    f32 = torch.float32
    args = PolicyArgs(_vector(tokens, rows, torch.int64, logits, "tokens"),
                      _vector(offsets, sequences + 1, torch.int64, logits, "offsets"),
                      _vector(old_logprob, rows, f32, logits, "old_logprob"),
                      None if ref_logprob is None else _vector(ref_logprob, rows, f32, logits, "ref_logprob"),
                      _vector(advantage, rows if advantage_per_token else sequences, f32, logits, "advantage"),
                      sequences, bool(advantage_per_token), REDUCTIONS[reduction], clip_low, clip_high, kl_coef,
                      entropy_coef, temperature, grad_scale)
    lib = load()
    with _allocate(stream):
        g = _grad_like(logits, out, grad)
        stats = torch.empty(POLICY_STATS, dtype=f32, device=logits.device)
        logprob = torch.empty(rows, dtype=f32, device=logits.device)
        work = _workspace("bf_policy_loss_workspace", rows, sequences, logits.device)
    _check(lib.bf_policy_loss(x, args, stats.data_ptr(), logprob.data_ptr(), None if g is None else _matrix(g, "out"),
                              work.data_ptr(), work.numel(), _stream_of(stream, logits)))
    _written(out if grad else None)
    return PolicyLoss(stats, logprob, g)


def preference_loss(logits, tokens, offsets, ref_logprob=None, *, beta: float = 0.1, label_smoothing: float = 0.0,
                    margin: float = 0.0, average: bool = False, temperature: float = 1.0, grad_scale: float = 1.0,
                    grad: bool = True, out=None, stream=None) -> PreferenceLoss:
    """The preference loss over pairs of answers (sequence 2p of `offsets` is preferred to 2p + 1) and its gradient in
    the logits (times `grad_scale`).  `out` may be `logits`: the gradient then replaces them."""
    import torch
    x = _matrix(logits, "logits")
    rows, pairs = x.rows, offsets.numel() // 2
    if offsets.numel() % 2 == 0:
        raise ValueError("offsets must hold 2 * pairs + 1 elements")
    f32 = torch.float32
    args = PreferenceArgs(_vector(tokens, rows, torch.int64, logits, "tokens"),
                          _vector(offsets, 2 * pairs + 1, torch.int64, logits, "offsets"),
                          None if ref_logprob is None else _vector(ref_logprob, rows, f32, logits, "ref_logprob"),
                          pairs, bool(average), beta, label_smoothing, margin, temperature, grad_scale)
    lib = load()
    with _allocate(stream):
        g = _grad_like(logits, out, grad)
        stats = torch.empty(PREFERENCE_STATS, dtype=f32, device=logits.device)
        rewards = torch.empty(2 * pairs, dtype=f32, device=logits.device)
        logprob = torch.empty(rows, dtype=f32, device=logits.device)
        work = _workspace("bf_preference_loss_workspace", rows, pairs, logits.device)
    _check(lib.bf_preference_loss(x, args, stats.data_ptr(), rewards.data_ptr(), logprob.data_ptr(),
                                  None if g is None else _matrix(g, "out"), work.data_ptr(), work.numel(),
                                  _stream_of(stream, logits)))
    _written(out if grad else None)
    return PreferenceLoss(stats, rewards, logprob, g)


def embed(table, tokens, *, scale: float = 1.0, out=None, stream=None):
    """Rows scale * table[tokens] (zeros for a token below 0), one per token of the 1-D int64 tensor."""
    import torch
    w = _matrix(table, "table")
    y = _vector(tokens, tokens.numel(), torch.int64, table, "tokens")
    given = out
    with _allocate(stream):
        if out is None:
            out = torch.empty(tokens.numel(), w.cols, dtype=table.dtype, device=table.device)
    o = _matrix(out, "out")
    if o.rows != tokens.numel():
        raise ValueError("out must have one row per token")
    _check(load().bf_embed(w, y, scale, o, _stream_of(stream, table)))
    _written(given)
    return out


def embed_grad(grad_out, tokens, vocab: int, *, scale: float = 1.0, out=None, accumulate: bool = False, stream=None):
    """The gradient of :func:`embed` in its table (vocab x width): scale * the sums of `grad_out`'s rows by token, of
    grad_out's type or in `out` (any of the types); with ``accumulate`` added to what `out` holds."""
    import torch
    g = _matrix(grad_out, "grad_out")
    y = _vector(tokens, g.rows, torch.int64, grad_out, "tokens")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    lib, given = load(), out
    with _allocate(stream):
        if out is None:
            out = torch.empty(vocab, g.cols, dtype=grad_out.dtype, device=grad_out.device)
        work = _workspace("bf_embed_grad_workspace", g.rows, g.cols, grad_out.device)
    o = _matrix(out, "out")
    if o.rows != vocab:
        raise ValueError("out must have one row per token of the vocabulary")
    _check(lib.bf_embed_grad(g, y, scale, accumulate, o, work.data_ptr(), work.numel(), _stream_of(stream, grad_out)))
    _written(given)
    return out


# ---- answering ------------------------------------------------------------------------------------------------------

MAX_BEAMS, MAX_STATES = 256, 128


class BeamStep(NamedTuple):
    """The continuations kept, the best first (each groups x keep): ``scores`` (float32), ``tokens`` and ``parents``
    (int64; a parent is a row of the logits), ``finished`` (bool) and, where lengths were given, ``lengths`` (int64)."""
    scores: object
    tokens: object
    parents: object
    finished: object
    lengths: object


class AttentionCall(ctypes.Structure):
    """What a call of ``bf_prefix_attention`` reads, in one piece."""
    _fields_ = [("caches", Cache * 6), ("args", AttentionArgs)]  # q, prefix_k, prefix_v, suffix_k, suffix_v, out


# Where the caches (their addresses first) and the arguments (the lengths' first) are in it, in words.
_DATA = tuple(i * ctypes.sizeof(Cache) // 8 for i in range(6)) + (AttentionCall.args.offset // 8,)


def _check_vectors(shape, stride, dtype, name: str, dims: int) -> None:
    if _dtype_code(dtype) is None or len(shape) != dims:
        raise ValueError(f"{name} must be a {dims}-D CUDA tensor of float32, bfloat16 or float16")
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must have contiguous vectors")


@functools.lru_cache(maxsize=256)
def _attention_call(shapes, strides, dtypes, scale: Optional[float]):
    """The parts of a call that only shapes, strides and types decide: (AttentionCall without addresses, bytes of
    workspace).  The last of the tensors is the output (None: contiguous, as the queries); suffixes may be missing."""
    names = ("q", "prefix_k", "prefix_v", "suffix_k", "suffix_v", "out")
    for shape, stride, dtype, name in zip(shapes, strides, dtypes, names):
        if shape is not None:
            _check_vectors(shape, stride, dtype, name, 3 if name in ("q", "out") else 4)
    call = AttentionCall()
    if shapes[5] is None:
        shapes = (*shapes[:5], shapes[0])
        strides = (*strides[:5], (shapes[0][1] * shapes[0][2], shapes[0][2], 1))
        dtypes = (*dtypes[:5], dtypes[0])
    for c, shape, stride, dtype in zip(call.caches, shapes, strides, dtypes):
        if shape is not None:
            c.batch, c.heads, c.dim = shape[0], shape[-2], shape[-1]
            c.tokens, c.token_stride = (1, 0) if len(shape) == 3 else (shape[1], stride[1])
            c.batch_stride, c.head_stride, c.dtype = stride[0], stride[-2], _dtype_code(dtype)
    call.args.scale = max(1, shapes[0][2]) ** -0.5 if scale is None else scale
    # Sizes that are refused have no workspace: the call itself says why.
    probe = AttentionCall.from_buffer_copy(call)
    for c in probe.caches:
        c.data, c.batch_stride, c.token_stride, c.head_stride = 256, 0, 0, 0
    need = ctypes.c_uint64(0)
    at = [ctypes.addressof(c) for c in probe.caches]
    ok = load().bf_prefix_attention_workspace(at[0], at[1], None if shapes[3] is None else at[3], ctypes.byref(need)) == BF_OK
    return bytes(call), need.value if ok else 256


def prefix_attention(q, prefix_k, prefix_v, suffix_k=None, suffix_v=None, *, prefix_lengths=None, suffix_lengths=None,
                     scale: Optional[float] = None, lse: bool = False, out=None, stream=None):
    """Attention of one token of each answer, `q` (answers x heads x dim), to its prompt's keys and values, `prefix_k`
    and `prefix_v` (prompts x tokens x key heads x dim; the answers of a prompt follow one another and share it), and to
    its own, `suffix_k` and `suffix_v` (answers x tokens x key heads x dim, or None).  Lengths (int64, one per prompt and
    per answer) say how many tokens hold something, all of them by default.  ``scale``: 1 / sqrt(dim) by default.
    Returns the outputs, of q's shape and type -- with ``lse``, the pair of them and the float32 logarithms of the sums
    of exponentials (answers x heads), by which a caller joins them with attention to other keys."""
    import torch
    tensors = (q, prefix_k, prefix_v, suffix_k, suffix_v, out)
    made, need = _attention_call(tuple([None if t is None else t.shape for t in tensors]),
                                 tuple([None if t is None else t.stride() for t in tensors]),
                                 tuple([None if t is None else t.dtype for t in tensors]), scale)
    current = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != current:
            raise ValueError(f"a tensor is on {t.device} but device {torch.cuda.current_device()} is current")
    i64 = torch.int64
    pl = None if prefix_lengths is None else _vector(prefix_lengths, prefix_k.shape[0], i64, q, "prefix_lengths")
    sl = None if suffix_lengths is None else _vector(suffix_lengths, q.shape[0], i64, q, "suffix_lengths")
    if sl is not None and suffix_k is None:
        raise ValueError("suffix_lengths needs suffix_k")
    given = out
    with _allocate(stream):
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        sums = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if lse else None
        work = torch.empty(need, dtype=torch.uint8, device=q.device)
    call = bytearray(made)
    words = memoryview(call).cast("Q")
    words[_DATA[0]], words[_DATA[1]], words[_DATA[2]] = q.data_ptr(), prefix_k.data_ptr(), prefix_v.data_ptr()
    if suffix_k is not None:
        words[_DATA[3]] = suffix_k.data_ptr()
    if suffix_v is not None:
        words[_DATA[4]] = suffix_v.data_ptr()
    words[_DATA[5]] = out.data_ptr()
    words[_DATA[6]], words[_DATA[6] + 1] = pl or 0, sl or 0
    at = ctypes.addressof(ctypes.c_char.from_buffer(call))
    _check(load().bf_prefix_attention(at, at + 8 * _DATA[1], at + 8 * _DATA[2], None if suffix_k is None else at + 8 * _DATA[3],
                                      None if suffix_v is None else at + 8 * _DATA[4], at + 8 * _DATA[6], at + 8 * _DATA[5],
                                      sums.data_ptr() if lse else None, work.data_ptr(), need, _stream_of(stream, q)))
    _written(given)
    return (out, sums) if lse else out


class BeamCall(ctypes.Structure):
    """What a call of ``bf_beam_step`` reads, in one piece."""
    _fields_ = [("logits", Matrix), ("args", BeamArgs)]


_BEAM_ARGS = BeamCall.args.offset // 8


@functools.lru_cache(maxsize=256)
def _beam_call(shape, stride, dtype, beams: int, keep: int, end_token: int, penalty: float, temperature: float):
    """The parts of a call that do not hold addresses: (BeamCall without them, groups, bytes of workspace)."""
    code = _dtype_code(dtype)
    if code is None or len(shape) != 2:
        raise ValueError("logits must be a 2-D CUDA tensor of float32, bfloat16 or float16")
    rows, cols = shape
    if stride[1] != 1 and cols > 1 and rows:
        raise ValueError("logits must have contiguous rows")
    if not 1 <= beams <= MAX_BEAMS or rows % beams:
        raise ValueError(f"beams must be 1 to {MAX_BEAMS} and a divisor of the rows")
    groups = rows // beams
    x = Matrix(None, rows, cols, max(stride[0], cols) if rows <= 1 else stride[0], code, 0)
    need = ctypes.c_uint64(0)
    _check(load().bf_beam_step_workspace(groups, beams, cols, keep, ctypes.byref(need)))
    return (bytes(BeamCall(x, BeamArgs(None, None, None, groups, beams, keep, end_token, penalty, temperature))), groups,
            need.value)


def beam_step(logits, scores, beams: int, *, keep: Optional[int] = None, finished=None, lengths=None,
              length_penalty: float = 0.0, end_token: int = -1, temperature: float = 1.0, stream=None) -> BeamStep:
    """The best `keep` (by default `beams`) continuations of every group of `beams` rows of `logits` (rows x vocab),
    by the beams' `scores` (float32, one per row; -inf: not alive) plus the tokens' log-probabilities.  A beam that is
    `finished` (bool, one per row) stays, with `end_token`.  With ``length_penalty`` (up to 65,536) continuations are ranked by score /
    length ** length_penalty, from the beams' `lengths` (int64, one per row).  Places without a continuation have score
    -inf and token -1."""
    import torch
    keep = beams if keep is None else keep
    made, groups, need = _beam_call(logits.shape, logits.stride(), logits.dtype, beams, keep, end_token, length_penalty, temperature)
    if logits.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"logits is on {logits.device} but device {torch.cuda.current_device()} is current")
    rows, device, i64 = logits.shape[0], logits.device, torch.int64
    call = bytearray(made)
    words = memoryview(call).cast("Q")
    words[0] = logits.data_ptr()
    words[_BEAM_ARGS] = _vector(scores, rows, torch.float32, logits, "scores")
    if finished is not None:
        words[_BEAM_ARGS + 1] = _vector(finished, rows, torch.bool, logits, "finished")
    if lengths is not None:
        words[_BEAM_ARGS + 2] = _vector(lengths, rows, i64, logits, "lengths")
    with _allocate(stream):
        best = torch.empty(groups, keep, dtype=torch.float32, device=device)
        whole = torch.empty(2 if lengths is None else 3, groups, keep, dtype=i64, device=device)
        ended = torch.empty(groups, keep, dtype=torch.bool, device=device)
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    at, to, step = ctypes.addressof(ctypes.c_char.from_buffer(call)), whole.data_ptr(), 8 * groups * keep
    _check(load().bf_beam_step(at, at + 8 * _BEAM_ARGS, best.data_ptr(), to, to + step, ended.data_ptr(),
                               None if lengths is None else to + 2 * step, work.data_ptr() if need else None, need,
                               _stream_of(stream, logits)))
    tokens, parents, *more = whole.unbind(0)
    return BeamStep(best, tokens, parents, ended, more[0] if more else None)


def _addresses(tensors, name: str):
    """The addresses of tensors of one layout (rows x tokens x ...) on the current device."""
    import torch
    first = tensors[0]
    shape, stride, dtype, current = first.shape, first.stride(), first.dtype, torch._C._cuda_getDevice()
    if len(shape) < 2:
        raise ValueError(f"{name} must have rows and tokens")
    for t in tensors:
        if t.shape != shape or t.stride() != stride or t.dtype != dtype or not t.is_cuda:
            raise ValueError(f"{name} must be CUDA tensors of one shape, layout and type")
        if t.get_device() != current:
            raise ValueError(f"{name} is on device {t.get_device()} but device {current} is current")
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def _layouts(source, target):
    """``bf_states`` of two tensors of one shape: what follows a token is runs that are contiguous in both, and at most
    one dimension that is apart."""
    shape, size = source.shape, source.element_size()
    strides = source.stride(), target.stride()
    dims = [(n, s, t) for n, s, t in zip(shape[2:], strides[0][2:], strides[1][2:]) if n != 1]
    width = 1
    while dims and dims[-1][1] == width == dims[-1][2]:
        width *= dims.pop()[0]
    heads, apart = 1, (0, 0)
    if dims and width:
        heads, *apart = dims.pop()
        while dims and dims[-1][1] == heads * apart[0] and dims[-1][2] == heads * apart[1]:
            heads *= dims.pop()[0]
        if dims:
            raise ValueError("states and out have more than one dimension apart behind their tokens")
    return [States(shape[0], shape[1], heads, width * size, s[0] * size, s[1] * size, a * size) for s, a in zip(strides, apart)]


def beam_reorder(states, parents, beams: int, *, lengths=None, out=None, stream=None):
    """Row i of each of `states` (a tensor rows x tokens x ..., or a list of up to MAX_STATES of one layout: caches,
    histories) takes row parents[i] (int64, within its group of `beams` rows), in place or in `out`.  `lengths` (int64,
    one per row): how many tokens a parent's row holds, of which the others are not written; all of them by default.
    Returns `states` or `out`."""
    import torch
    one = not isinstance(states, (list, tuple))
    source = [states] if one else states
    target = source if out is None else [out] if one else out
    if not source:
        return states if out is None else out
    if len(source) > MAX_STATES or len(target) != len(source) or target[0].dtype != source[0].dtype:
        raise ValueError(f"states must be up to {MAX_STATES} tensors, and out as many of their type")
    like = source[0]
    from_ = _addresses(source, "states")
    to = from_ if out is None else _addresses(target, "out")
    if target[0].shape != like.shape:
        raise ValueError("out must have the shape of states")
    layout, to_layout = _layouts(like, target[0])
    y = _vector(parents, layout.rows, torch.int64, like, "parents")
    n = None if lengths is None else _vector(lengths, layout.rows, torch.int64, like, "lengths")
    _check(load().bf_beam_reorder(from_, layout, to, to_layout, len(source), y, beams, n, _stream_of(stream, like)))
    for t in target:
        _written(t)
    return states if out is None else out
