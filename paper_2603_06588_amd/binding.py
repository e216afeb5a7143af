"""ctypes front end of libhook.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
``include/hook_api.h``; torch is used for device memory and the current stream.
There is no CPU fallback: loading fails loudly if the library has not been
built (``python -m paper_2603_06588_amd.build``).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhook.so")

HOOK_OK = 0
HOOK_BF16, HOOK_F32 = 0, 1
_DT = {torch.bfloat16: HOOK_BF16, torch.float32: HOOK_F32}
EXPORTS = ["hook_attn_probe_workspace_bytes", "hook_attn_probe", "hook_attn_probe_static", "hook_attn_probe_static_capacity",
           "hook_attn_probe_device_status", "hook_attn_probe_validate", "hook_span_mass", "hook_span_mass_workspace_bytes",
           "hook_steer", "hook_residual_add_steer", "hook_kv_write", "hook_capture_qk", "hook_reduce_mass", "hook_parse_layer_heads", "hook_parse_config_json", "hook_status_string", "hook_version",
           "hook_rope", "hook_pages_workspace_bytes", "hook_pages_fork", "hook_pages_append", "hook_pages_compact", "hook_steer_logits"]


class HookAttnProbeArgs(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("total_q", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32), ("num_blocks", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("q", ctypes.c_void_p), ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
        ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
        ("num_probe_heads", ctypes.c_int32), ("probe_heads", ctypes.c_void_p),
        ("max_sel_q", ctypes.c_int32), ("query_sel", ctypes.c_void_p),
        ("max_spans", ctypes.c_int32), ("key_spans", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("mass", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p), ("batch_kind", ctypes.c_int32), ("plan_mode", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p),
    ]


class HookCaptureQkArgs(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("total_q", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32), ("num_blocks", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("k_cache", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
        ("seq_lens", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
        ("num_probe_heads", ctypes.c_int32), ("probe_heads", ctypes.c_void_p),
        ("max_sel_q", ctypes.c_int32), ("query_sel", ctypes.c_void_p),
        ("num_capture_kv_heads", ctypes.c_int32), ("capture_kv_heads", ctypes.c_void_p),
        ("cu_k_lens", ctypes.c_void_p), ("total_k", ctypes.c_int32),
        ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p), ("stream", ctypes.c_void_p),
        ("kv_dtype", ctypes.c_int32),
    ]


class HookKvWriteArgs(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("total_q", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32),
        ("num_blocks", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
        ("seq_lens", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
        ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("stream", ctypes.c_void_p),
        ("kv_dtype", ctypes.c_int32), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
    ]


class HookReduceArgs(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("num_probe_heads", ctypes.c_int32), ("max_sel_q", ctypes.c_int32),
        ("max_spans", ctypes.c_int32),
        ("mass", ctypes.c_void_p), ("query_sel", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
        ("head_weights", ctypes.c_void_p),
        ("mode", ctypes.c_int32), ("span_a", ctypes.c_int32), ("span_b", ctypes.c_int32),
        ("accumulate", ctypes.c_int32),
        ("scores", ctypes.c_void_p), ("stream", ctypes.c_void_p),
    ]


class HookRopeArgs(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("num_axes", ctypes.c_int32),
        ("axis_pairs", ctypes.c_int32 * 4), ("layout", ctypes.c_int32), ("axis_order", ctypes.c_int32),
        ("inverse", ctypes.c_int32), ("dtype", ctypes.c_int32), ("magnitude", ctypes.c_float),
        ("positions", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64),
        ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64),
        ("num_seqs", ctypes.c_int32), ("block_size", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32),
        ("num_blocks", ctypes.c_int32), ("v", ctypes.c_void_p), ("v_stride", ctypes.c_int64),
        ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
        ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("kv_dtype", ctypes.c_int32),
        ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("stream", ctypes.c_void_p),
    ]


class HookPagesArgs(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32), ("num_blocks", ctypes.c_int32),
        ("block_size", ctypes.c_int32), ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
        ("ref_counts", ctypes.c_void_p), ("block_table_out", ctypes.c_void_p), ("seq_lens_out", ctypes.c_void_p),
        ("ref_counts_out", ctypes.c_void_p), ("status", ctypes.c_void_p), ("num_rows", ctypes.c_int32),
        ("src_rows", ctypes.c_void_p), ("src_lens", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
        ("page_map", ctypes.c_void_p), ("num_live", ctypes.c_void_p), ("num_caches", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("row_bytes", ctypes.c_int64), ("caches", ctypes.POINTER(ctypes.c_void_p)),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p),
    ]


class HookSteerLogitsArgs(ctypes.Structure):
    _fields_ = [
        ("num_rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("logits", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("logits_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
        ("history_len", ctypes.c_int32), ("history", ctypes.c_void_p), ("cu_history", ctypes.c_void_p),
        ("prompt_lens", ctypes.c_void_p), ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
        ("presence", ctypes.c_void_p), ("bias_len", ctypes.c_int32), ("cu_bias", ctypes.c_void_p),
        ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p), ("num_masks", ctypes.c_int32),
        ("mask", ctypes.c_void_p), ("mask_rows", ctypes.c_void_p), ("stream", ctypes.c_void_p),
    ]


REDUCE_SPAN_MEAN, REDUCE_RATIO_MEAN, REDUCE_RATIO_OF_SUMS = 0, 1, 2
BATCH_MIXED, BATCH_PREFILL_ONLY, BATCH_DECODE_ONLY = 0, 1, 2
KV_SAME, KV_FP8_E4M3 = 0, 1
PLAN_FRESH, PLAN_REUSE = 0, 1
(BAD_ROWS_EXCEED_CONTEXT, BAD_CONTEXT_TOO_LONG, BAD_LENGTH, BAD_BATCH_KIND, BAD_BLOCK_ID, BAD_PROBE_HEADS,
 BAD_QUERY_SEL) = 1, 2, 4, 8, 16, 32, 64
ROPE_HALVES, ROPE_NEIGHBOURS = 0, 1
ROPE_BLOCKED, ROPE_CYCLIC = 0, 1
PAGES_FULL, PAGES_BAD_ROW, PAGES_BAD_LENGTH, PAGES_BAD_PAGE = 1, 2, 4, 8


class HookError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {status_string(status)} (hook_status {int(status)})")


_lib = None


def load_library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_06588_amd.build` "
                               "(there is no fallback path)")
        lib = ctypes.CDLL(LIB_PATH)
        ap = ctypes.POINTER(HookAttnProbeArgs)
        lib.hook_attn_probe_workspace_bytes.restype = ctypes.c_size_t
        lib.hook_attn_probe_workspace_bytes.argtypes = [ap]
        lib.hook_attn_probe.restype = ctypes.c_int
        lib.hook_attn_probe.argtypes = [ap]
        lib.hook_attn_probe_static.restype = ctypes.c_int
        lib.hook_attn_probe_static.argtypes = [ap]
        lib.hook_attn_probe_static_capacity.restype = ctypes.c_size_t
        lib.hook_attn_probe_static_capacity.argtypes = []
        lib.hook_attn_probe_device_status.restype = ctypes.c_int
        lib.hook_attn_probe_device_status.argtypes = [ctypes.c_void_p, ctypes.c_void_p,
                                                      ctypes.POINTER(ctypes.c_int32)]
        lib.hook_attn_probe_validate.restype = ctypes.c_int
        lib.hook_attn_probe_validate.argtypes = [ap, ctypes.POINTER(ctypes.c_int32)]
        lib.hook_steer.restype = ctypes.c_int
        lib.hook_steer.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p,
                                   ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]
        lib.hook_capture_qk.restype = ctypes.c_int
        lib.hook_capture_qk.argtypes = [ctypes.POINTER(HookCaptureQkArgs)]
        lib.hook_kv_write.restype = ctypes.c_int
        lib.hook_kv_write.argtypes = [ctypes.POINTER(HookKvWriteArgs)]
        lib.hook_span_mass_workspace_bytes.restype = ctypes.c_size_t
        lib.hook_span_mass_workspace_bytes.argtypes = [ctypes.POINTER(HookAttnProbeArgs)]
        lib.hook_span_mass.restype = ctypes.c_int
        lib.hook_span_mass.argtypes = [ctypes.POINTER(HookAttnProbeArgs)]
        lib.hook_residual_add_steer.restype = ctypes.c_int
        lib.hook_residual_add_steer.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                                                ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                                ctypes.c_void_p]
        lib.hook_reduce_mass.restype = ctypes.c_int
        lib.hook_reduce_mass.argtypes = [ctypes.POINTER(HookReduceArgs)]
        lib.hook_parse_layer_heads.restype = ctypes.c_int
        lib.hook_parse_layer_heads.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_int32),
                                               ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                               ctypes.POINTER(ctypes.c_int32)]
        lib.hook_parse_config_json.restype = ctypes.c_int
        lib.hook_parse_config_json.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_int32),
                                               ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                               ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        lib.hook_rope.restype = ctypes.c_int
        lib.hook_rope.argtypes = [ctypes.POINTER(HookRopeArgs)]
        pp = ctypes.POINTER(HookPagesArgs)
        lib.hook_pages_workspace_bytes.restype = ctypes.c_size_t
        lib.hook_pages_workspace_bytes.argtypes = [pp]
        for fn in (lib.hook_pages_fork, lib.hook_pages_append, lib.hook_pages_compact):
            fn.restype = ctypes.c_int
            fn.argtypes = [pp]
        lib.hook_steer_logits.restype = ctypes.c_int
        lib.hook_steer_logits.argtypes = [ctypes.POINTER(HookSteerLogitsArgs)]
        lib.hook_status_string.restype = ctypes.c_char_p
        lib.hook_status_string.argtypes = [ctypes.c_int]
        lib.hook_version.restype = ctypes.c_int
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load_library().hook_status_string(int(status)).decode()


def version() -> int:
    return int(load_library().hook_version())


def _p(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None or t.numel() == 0 else t.data_ptr()


def _stream_handle(stream) -> int:
    if stream is None:      # the current stream's handle itself: building a Stream object takes ten times as long
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


_SAME = contextlib.nullcontext()


def _taken_on(stream, device):
    """Where a call on `stream` takes new memory of `device` from: that stream's own pool.  A block of another stream's may be one that has just been given
    back there while work queued on it still uses the block, and nothing orders the call behind that work."""
    if stream is None:
        return _SAME
    # (another program's stream, known by its handle alone, will do)
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream.cuda_stream), device=device))


def _handed_over(stream, *results):
    """Results that a call on `stream` has taken memory for are read on the current stream (once the program has made it wait): their
    memory is not given to anybody else before that is done."""
    if stream is not None and results:
        current = torch.cuda.current_stream(results[0].device)
        if current.cuda_stream != int(stream.cuda_stream):
            for t in results:
                t.record_stream(current)


class AttnProbeCall:
    """A marshalled ``hook_attn_probe`` call that can be launched repeatedly.

    Holds references to every tensor it points at, the output tensors and the
    workspace, so relaunching costs one ctypes call and no allocation.  What it
    allocates belongs to the stream that is current where it is made: a launch on
    another stream waits for that one first, and the object outlives the launch.
    """

    def __init__(self, q, k_cache, v_cache, block_table, seq_lens, cu_q_lens, probe_heads=None, max_sel_q=1,
                 query_sel=None, max_spans=1, key_spans=None, scale: float = 0.0, out=None, mass=None,
                 workspace=None, batch_kind: int = 0, plan_mode: int = 0, k_scale=None, v_scale=None,
                 k_new=None, v_new=None):
        lib = load_library()
        if q.dtype not in _DT:
            raise HookError(3, "hook_attn_probe (dtype)")
        dev = q.device
        self.keep = [q, k_cache, v_cache, block_table, seq_lens, cu_q_lens, probe_heads, query_sel, key_spans,
                     k_scale, v_scale, k_new, v_new]
        total_q, Hq, d = q.shape
        num_blocks, Hkv, B, _ = k_cache.shape
        num_seqs, max_blocks = block_table.shape
        P = 0 if probe_heads is None else int(probe_heads.numel())
        a = HookAttnProbeArgs()
        a.num_seqs, a.total_q, a.num_q_heads, a.num_kv_heads = num_seqs, total_q, Hq, Hkv
        a.head_dim, a.block_size, a.max_blocks_per_seq, a.num_blocks = d, B, max_blocks, num_blocks
        a.dtype, a.scale = _DT[q.dtype], float(scale)
        a.q, a.k_cache, a.v_cache = _p(q), _p(k_cache), _p(v_cache)
        a.block_table, a.seq_lens, a.cu_q_lens = _p(block_table), _p(seq_lens), _p(cu_q_lens)
        a.num_probe_heads, a.probe_heads = P, _p(probe_heads)
        a.max_sel_q, a.query_sel = int(max_sel_q), _p(query_sel)
        a.max_spans, a.key_spans = int(max_spans), _p(key_spans)
        self.out = out if out is not None else torch.empty_like(q)
        self.mass = mass if mass is not None else torch.empty((num_seqs, P, int(max_sel_q), int(max_spans)),
                                                               dtype=torch.float32, device=dev)
        a.out, a.mass = _p(self.out), _p(self.mass)
        need = int(lib.hook_attn_probe_workspace_bytes(ctypes.byref(a)))
        if workspace is None:
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        self.workspace = workspace
        a.workspace, a.workspace_bytes = _p(workspace), workspace.numel()
        a.batch_kind = int(batch_kind)
        a.plan_mode = int(plan_mode)
        if k_cache.dtype == torch.uint8:      # 8-bit E4M3 bytes with one scale per kv head
            a.kv_dtype, a.k_scale, a.v_scale = KV_FP8_E4M3, _p(k_scale), _p(v_scale)
        a.k_new, a.v_new = _p(k_new), _p(v_new)
        self.args = a
        self.workspace_needed = need
        self._fn = lib.hook_attn_probe

    def launch(self, stream=None) -> None:
        self.args.stream = _stream_handle(stream)
        st = self._fn(ctypes.byref(self.args))
        if st != HOOK_OK:
            raise HookError(st, "hook_attn_probe")

    def launch_static(self, stream=None) -> None:
        """The same call on the library's own scratch array (the workspace of this object is not used)."""
        self.args.stream = _stream_handle(stream)
        st = load_library().hook_attn_probe_static(ctypes.byref(self.args))
        if st != HOOK_OK:
            raise HookError(st, "hook_attn_probe_static")

    def device_status(self, stream=None) -> int:
        bits = ctypes.c_int32(0)
        st = load_library().hook_attn_probe_device_status(self.args.workspace, _stream_handle(stream),
                                                          ctypes.byref(bits))
        if st != HOOK_OK:
            raise HookError(st, "hook_attn_probe_device_status")
        return int(bits.value)

    def validate(self, stream=None) -> int:
        """Problem bits (HOOK_BAD_*) of the device-resident contents of this call; synchronises."""
        bits = ctypes.c_int32(0)
        self.args.stream = _stream_handle(stream)
        st = load_library().hook_attn_probe_validate(ctypes.byref(self.args), ctypes.byref(bits))
        if st != HOOK_OK:
            raise HookError(st, "hook_attn_probe_validate")
        return int(bits.value)


def hook_attn_probe(q, k_cache, v_cache, block_table, seq_lens, cu_q_lens, probe_heads=None, max_sel_q=1,
                    query_sel=None, max_spans=1, key_spans=None, scale: float = 0.0,
                    stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(out, mass) of one layer's hooked attention; asynchronous on the current stream."""
    with _taken_on(stream, q.device):
        call = AttnProbeCall(q, k_cache, v_cache, block_table, seq_lens, cu_q_lens, probe_heads, max_sel_q,
                             query_sel, max_spans, key_spans, scale)
    call.launch(stream)
    _handed_over(stream, call.out, call.mass)
    return call.out, call.mass


def hook_span_mass(q, k_cache, block_table, seq_lens, cu_q_lens, probe_heads, max_sel_q, query_sel, max_spans,
                   key_spans, scale: float = 0.0, mass=None, stream=None, workspace=None,
                   use_workspace: bool = True, k_scale=None) -> torch.Tensor:
    """mass [num_seqs, P, NQ, S] for up to HOOK_MAX_SPANS_WIDE spans; computes no attention output.
    A scratch tensor lets the library split the work over the chip; it is allocated here unless
    one is passed in or use_workspace is False."""
    lib = load_library()
    total_q, Hq, d = q.shape
    num_blocks, Hkv, B, _ = k_cache.shape
    num_seqs, max_blocks = block_table.shape
    P = int(probe_heads.numel())
    if q.dtype not in _DT:
        raise HookError(3, "hook_span_mass (dtype)")
    results = ()
    if mass is None:
        with _taken_on(stream, q.device):
            mass = torch.empty((num_seqs, P, int(max_sel_q), int(max_spans)), dtype=torch.float32, device=q.device)
        results = (mass,)
    a = HookAttnProbeArgs()
    a.num_seqs, a.total_q, a.num_q_heads, a.num_kv_heads = num_seqs, total_q, Hq, Hkv
    a.head_dim, a.block_size, a.max_blocks_per_seq, a.num_blocks = d, B, max_blocks, num_blocks
    a.dtype, a.scale = _DT[q.dtype], float(scale)
    a.q, a.k_cache = _p(q), _p(k_cache)
    a.block_table, a.seq_lens, a.cu_q_lens = _p(block_table), _p(seq_lens), _p(cu_q_lens)
    a.num_probe_heads, a.probe_heads = P, _p(probe_heads)
    a.max_sel_q, a.query_sel = int(max_sel_q), _p(query_sel)
    a.max_spans, a.key_spans = int(max_spans), _p(key_spans)
    a.mass, a.stream = _p(mass), _stream_handle(stream)
    if k_cache.dtype == torch.uint8:          # 8-bit E4M3 bytes with one scale per kv head
        a.kv_dtype, a.k_scale = KV_FP8_E4M3, _p(k_scale)
    if workspace is None and use_workspace:
        need = int(lib.hook_span_mass_workspace_bytes(ctypes.byref(a)))
        with _taken_on(stream, q.device):
            workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=q.device) if need else None
    if workspace is not None:
        a.workspace, a.workspace_bytes = _p(workspace), workspace.numel()
    st = lib.hook_span_mass(ctypes.byref(a))
    if st != HOOK_OK:
        raise HookError(st, "hook_span_mass")
    _handed_over(stream, *results)
    return mass


def hook_span_mass_batch(b, stream=None, mass=None, workspace=None, use_workspace: bool = True) -> torch.Tensor:
    return hook_span_mass(b.q, b.k_cache, b.block_table, b.seq_lens, b.cu_q_lens, b.probe_heads, b.max_sel_q,
                          b.query_sel, b.max_spans, b.key_spans, b.scale, mass, stream, workspace, use_workspace,
                          k_scale=getattr(b, "k_scale", None))


def hook_attn_probe_batch(b, stream=None, probe: bool = True):
    """Convenience for objects carrying the batch attributes (device tensors)."""
    return hook_attn_probe(b.q, b.k_cache, b.v_cache, b.block_table, b.seq_lens, b.cu_q_lens,
                           b.probe_heads if probe else None, b.max_sel_q, b.query_sel, b.max_spans,
                           b.key_spans, b.scale, stream)


def call_from_batch(b, probe: bool = True, **kw) -> AttnProbeCall:
    if getattr(b, "k_scale", None) is not None:
        kw.setdefault("k_scale", b.k_scale)
        kw.setdefault("v_scale", b.v_scale)
    return AttnProbeCall(b.q, b.k_cache, b.v_cache, b.block_table, b.seq_lens, b.cu_q_lens,
                         b.probe_heads if probe else None, b.max_sel_q, b.query_sel, b.max_spans,
                         b.key_spans, b.scale, **kw)


def hook_residual_add_steer(hidden, delta, vec, alpha: float, token_mask=None, stream=None):
    """hidden += delta (+ alpha * vec on masked rows), in place, one rounding."""
    lib = load_library()
    T, D = hidden.shape
    st = lib.hook_residual_add_steer(_p(hidden), _p(delta), _p(vec), float(alpha), _p(token_mask), T, D,
                                     _DT[hidden.dtype], _stream_handle(stream))
    if st != HOOK_OK:
        raise HookError(st, "hook_residual_add_steer")
    return hidden


def hook_kv_write(k_new, v_new, block_table, seq_lens, cu_q_lens, k_cache, v_cache, stream=None, k_scale=None,
                  v_scale=None) -> None:
    """Scatter the new tokens' K/V rows ([total_q, Hkv, d]) into the paged cache, in place (quantising
    when the cache is uint8 E4M3 bytes with per-kv-head scales)."""
    lib = load_library()
    total_q, Hkv, d = k_new.shape
    num_blocks, _, B, _ = k_cache.shape
    num_seqs, max_blocks = block_table.shape
    a = HookKvWriteArgs()
    a.num_seqs, a.total_q, a.num_kv_heads, a.head_dim = num_seqs, total_q, Hkv, d
    a.block_size, a.max_blocks_per_seq, a.num_blocks, a.dtype = B, max_blocks, num_blocks, _DT[k_new.dtype]
    a.k_new, a.v_new, a.block_table = _p(k_new), _p(v_new), _p(block_table)
    a.seq_lens, a.cu_q_lens = _p(seq_lens), _p(cu_q_lens)
    a.k_cache, a.v_cache, a.stream = _p(k_cache), _p(v_cache), _stream_handle(stream)
    if k_cache.dtype == torch.uint8:
        a.kv_dtype, a.k_scale, a.v_scale = KV_FP8_E4M3, _p(k_scale), _p(v_scale)
    st = lib.hook_kv_write(ctypes.byref(a))
    if st != HOOK_OK:
        raise HookError(st, "hook_kv_write")


def hook_capture_qk(q, k_cache, block_table, seq_lens, cu_q_lens, probe_heads, max_sel_q, query_sel,
                    capture_kv_heads, cu_k_lens, total_k: int, stream=None, q_out=None, k_out=None):
    """Gather (q_out [num_seqs, P, NQ, d], k_out [total_k, KH, d]); total_k is a host integer."""
    lib = load_library()
    total_q, Hq, d = q.shape
    num_blocks, Hkv, B, _ = k_cache.shape
    num_seqs, max_blocks = block_table.shape
    P = int(probe_heads.numel()) if probe_heads is not None else 0
    KH = int(capture_kv_heads.numel()) if capture_kv_heads is not None else 0
    results = []
    with _taken_on(stream, q.device):
        if q_out is None:
            q_out = torch.empty((num_seqs, P, int(max_sel_q), d), dtype=q.dtype, device=q.device)
            results.append(q_out)
        if k_out is None:
            k_out = torch.empty((int(total_k), KH, d), dtype=k_cache.dtype, device=q.device)   # bytes for an 8-bit cache
            results.append(k_out)
    a = HookCaptureQkArgs()
    a.num_seqs, a.total_q, a.num_q_heads, a.num_kv_heads = num_seqs, total_q, Hq, Hkv
    a.head_dim, a.block_size, a.max_blocks_per_seq, a.num_blocks = d, B, max_blocks, num_blocks
    a.dtype = _DT[q.dtype]
    a.q, a.k_cache, a.block_table = _p(q), _p(k_cache), _p(block_table)
    a.seq_lens, a.cu_q_lens = _p(seq_lens), _p(cu_q_lens)
    a.num_probe_heads, a.probe_heads, a.max_sel_q, a.query_sel = P, _p(probe_heads), int(max_sel_q), _p(query_sel)
    a.num_capture_kv_heads, a.capture_kv_heads = KH, _p(capture_kv_heads)
    a.cu_k_lens, a.total_k = _p(cu_k_lens), int(total_k)
    a.q_out, a.k_out, a.stream = _p(q_out), _p(k_out), _stream_handle(stream)
    a.kv_dtype = KV_FP8_E4M3 if k_cache.dtype == torch.uint8 else KV_SAME
    st = lib.hook_capture_qk(ctypes.byref(a))
    if st != HOOK_OK:
        raise HookError(st, "hook_capture_qk")
    _handed_over(stream, *results)
    return q_out, k_out


def hook_reduce_mass(mass, mode: int, span_a: int = 0, span_b: int = 1, query_sel=None, cu_q_lens=None,
                     head_weights=None, scores=None, accumulate: bool = False, stream=None):
    """Reduce mass [num_seqs, P, NQ, S] to scores ([num_seqs, S] for SPAN_MEAN, else [num_seqs])."""
    lib = load_library()
    num_seqs, P, NQ, S = mass.shape
    results = ()
    if scores is None:
        if accumulate:
            raise ValueError("accumulate needs an existing scores tensor")
        shape = (num_seqs, S) if mode == REDUCE_SPAN_MEAN else (num_seqs,)
        with _taken_on(stream, mass.device):
            scores = torch.empty(shape, dtype=torch.float32, device=mass.device)
        results = (scores,)
    a = HookReduceArgs()
    a.num_seqs, a.num_probe_heads, a.max_sel_q, a.max_spans = num_seqs, P, NQ, S
    a.mass, a.query_sel, a.cu_q_lens, a.head_weights = _p(mass), _p(query_sel), _p(cu_q_lens), _p(head_weights)
    a.mode, a.span_a, a.span_b, a.accumulate = int(mode), int(span_a), int(span_b), int(bool(accumulate))
    a.scores, a.stream = _p(scores), _stream_handle(stream)
    st = lib.hook_reduce_mass(ctypes.byref(a))
    if st != HOOK_OK:
        raise HookError(st, "hook_reduce_mass")
    _handed_over(stream, *results)
    return scores


def parse_layer_heads(text: str):
    """'0:0,3,6;15:2' -> [(0, 0), (0, 3), (0, 6), (15, 2)] (parsed by the library)."""
    lib = load_library()
    count = ctypes.c_int32(0)
    st = lib.hook_parse_layer_heads(text.encode(), None, None, 0, ctypes.byref(count))
    if st not in (HOOK_OK, 4):
        raise HookError(st, "hook_parse_layer_heads")
    n = int(count.value)
    layers, heads = (ctypes.c_int32 * max(n, 1))(), (ctypes.c_int32 * max(n, 1))()
    st = lib.hook_parse_layer_heads(text.encode(), layers, heads, n, ctypes.byref(count))
    if st != HOOK_OK:
        raise HookError(st, "hook_parse_layer_heads")
    return [(int(layers[i]), int(heads[i])) for i in range(n)]


def parse_config_json(text: str):
    """JSON config text -> ([(layer, head), ...] in file order, hookq_mode or None)."""
    lib = load_library()
    count, mode = ctypes.c_int32(0), ctypes.c_int32(-1)
    st = lib.hook_parse_config_json(text.encode(), None, None, 0, ctypes.byref(count), ctypes.byref(mode))
    if st not in (HOOK_OK, 4):
        raise HookError(st, "hook_parse_config_json")
    n = int(count.value)
    layers, heads = (ctypes.c_int32 * max(n, 1))(), (ctypes.c_int32 * max(n, 1))()
    st = lib.hook_parse_config_json(text.encode(), layers, heads, n, ctypes.byref(count), ctypes.byref(mode))
    if st != HOOK_OK:
        raise HookError(st, "hook_parse_config_json")
    names = {0: "last_token", 1: "all_tokens"}
    return [(int(layers[i]), int(heads[i])) for i in range(n)], names.get(int(mode.value))


def probe_heads_for_layer(pairs, layer: int, device="cpu") -> torch.Tensor:
    """Sorted, de-duplicated heads of one layer as the int32 probe_heads tensor of a call."""
    hs = sorted({int(h) for (l, h) in pairs if int(l) == int(layer)})
    return torch.tensor(hs, dtype=torch.int32, device=device)


def hook_steer(hidden: torch.Tensor, vec: torch.Tensor, alpha: float, token_mask: torch.Tensor,
               stream=None) -> torch.Tensor:
    """In place: hidden[t] += alpha * vec where token_mask[t] != 0.  Returns ``hidden``."""
    lib = load_library()
    if hidden.dtype not in _DT or vec.dtype != hidden.dtype or token_mask.dtype != torch.uint8:
        raise HookError(3, "hook_steer (dtype)")
    if not (hidden.is_contiguous() and vec.is_contiguous() and token_mask.is_contiguous()):
        raise HookError(2, "hook_steer (layout)")
    T, D = hidden.shape
    if vec.numel() != D or token_mask.numel() != T:
        raise HookError(2, "hook_steer (shape)")
    st = lib.hook_steer(_p(hidden), _p(vec), float(alpha), _p(token_mask), T, D, _DT[hidden.dtype],
                        _stream_handle(stream))
    if st != HOOK_OK:
        raise HookError(st, "hook_steer")
    return hidden


# The calls below run on small tensors too, where the host's time is what a call costs: all tensors of a call are looked at in one go
# (csrc/tensors.cpp: same GPU, types, layouts; an address and sizes for each), and the struct is filled in another.

_look_fn = None
_INT32_MAX = 0x7FFFFFFF      # sizes are 32 bits in the structs, which would take a larger one modulo 2^32


def _look(where: str, like, spec, *tensors):
    global _look_fn
    if _look_fn is None:
        if not os.path.exists(os.path.join(_HERE, "_tensors.so")):
            raise RuntimeError(f"{_HERE}/_tensors.so is missing: build it with `python -m paper_2603_06588_amd.build`")
        from . import _tensors
        _tensors.set_error(HookError)
        _look_fn = _tensors.look
    return _look_fn(where, like, spec, *tensors)


def _launch(fn, args, index: int, stream, where: str) -> None:
    """Launches on GPU `index`, which need not be the current one."""
    args.stream = torch._C._cuda_getCurrentRawStream(index) if stream is None else int(stream.cuda_stream)
    if index == torch._C._cuda_getDevice():
        st = fn(args)
    else:
        with torch.cuda.device(index):
            st = fn(args)
    if st != HOOK_OK:
        raise HookError(st, where)


_FourInts = ctypes.c_int32 * 4
_ROPE = ("rq", "rk", "rv", "rq_out", "rk_out", "ipositions", "finv_freq", "cblock_table", "iseq_lens", "icu_q_lens", "ck_cache", "cv_cache", "fk_scale",
         "fv_scale")


def hook_rope(q, k, positions, inv_freq, axis_pairs=None, layout: int = ROPE_HALVES, axis_order: int = ROPE_BLOCKED,
              inverse: bool = False, magnitude: float = 0.0, q_out=None, k_out=None, v=None, block_table=None, seq_lens=None,
              cu_q_lens=None, k_cache=None, v_cache=None, k_scale=None, v_scale=None, stream=None):
    """Turns q [T, Hq, d] and k [T, Hkv, d] by positions ([T] or [axes, T], int32) times inv_freq (fp32; twice as many elements of a
    head turn); either may be None.  In place where no output is given.  ``inverse`` with the same magnitude is the call's gradient, with
    one over it the way back.  With k_cache and v_cache the turned keys and v also
    go to the cache, as by ``hook_kv_write``; k itself is then left alone unless it is k_out.  Rows may be views into a wider
    buffer.  Returns (q_out, k_out)."""
    where = "hook_rope"
    if positions is None or inv_freq is None:      # (a head of which nothing turns has an empty inv_freq)
        raise HookError(1, "hook_rope (positions, inv_freq)")
    cached = k_cache is not None or v_cache is not None
    if q_out is None:
        q_out = q
    if k_out is None and not cached:
        k_out = k
    like = q if q is not None else k
    (index, qp, qs, qn, kp, ks, kn, vp, vs, vn, qop, qos, qon, kop, kos, kon, pos, npos, freq, pairs, table, tn, lens, nlens, cu, ncu, kc, kcn, vc, vcn,
     ksc, nks, vsc, nvs) = _look(where, like, _ROPE, q, k, v, q_out, k_out, positions, inv_freq, block_table, seq_lens, cu_q_lens, k_cache, v_cache,
                                 k_scale, v_scale)
    dt = like.dtype
    if dt not in _DT:
        raise HookError(3, "hook_rope (dtype)")
    shape = qn or kn
    if len(shape) != 3 or (kn and (len(kn) != 3 or kn[0] != shape[0] or kn[2] != shape[2])):
        raise HookError(2, "hook_rope (q, k: shape)")
    T, _, d = shape
    if qon != qn or (kon and kon != kn):
        raise HookError(2, "hook_rope (q_out, k_out: shape)")
    axes = positions.shape[0] if positions.dim() == 2 else 1
    if npos != axes * T:
        raise HookError(2, "hook_rope (positions: shape)")
    if axis_pairs is None:
        axis_pairs = (pairs,)
    if len(axis_pairs) != axes or axes > 4:
        raise HookError(2, "hook_rope (axis_pairs)")
    kv_dtype = num_seqs = block_size = max_blocks = num_blocks = 0
    if cached:
        if not kn or v is None or k_cache is None or v_cache is None or block_table is None or seq_lens is None or cu_q_lens is None:
            raise HookError(1, "hook_rope (cache)")
        if len(kcn) != 4 or kcn[1] != kn[1] or kcn[3] != d or vcn != kcn or vn != kn:
            raise HookError(2, "hook_rope (v, k_cache, v_cache: shape)")
        if len(tn) != 2 or nlens != tn[0] or ncu != nlens + 1:
            raise HookError(2, "hook_rope (block_table, seq_lens, cu_q_lens: shape)")
        kind = k_cache.dtype
        if v_cache.dtype is not kind or block_table.dtype is not torch.int32:
            raise HookError(3, "hook_rope (v_cache, block_table: dtype)")
        if kind is torch.uint8:       # 8-bit E4M3 bytes with one scale per kv head
            if nks != kn[1] or nvs != kn[1]:
                raise HookError(2, "hook_rope (k_scale, v_scale: shape)")
            kv_dtype = KV_FP8_E4M3
        elif kind is not dt:
            raise HookError(3, "hook_rope (k_cache: dtype)")
        num_seqs, max_blocks, num_blocks, block_size = nlens, tn[1], kcn[0], kcn[2]
    else:
        vp = table = lens = cu = 0
    hq, hkv = qn[1] if qn else 0, kn[1] if kn else 0
    if (T | hq | hkv | d | 2 * pairs | num_seqs | max_blocks | num_blocks | block_size) > _INT32_MAX:
        raise HookError(3, "hook_rope (sizes)")
    a = HookRopeArgs(T, hq, hkv, d, 2 * pairs, axes, _FourInts(*axis_pairs), layout, axis_order, 1 if inverse else 0,
                     _DT[dt], magnitude, pos, freq, qp, kp, qop, kop, qs, ks, qos, kos, num_seqs, block_size, max_blocks, num_blocks, vp, vs, table,
                     lens, cu, kc, vc, kv_dtype, ksc, vsc)
    _launch((_lib or load_library()).hook_rope, a, index, stream, where)
    return q_out, k_out


_PAGES = ("iblock_table", "iseq_lens", "iref_counts", "iblock_table_out", "iseq_lens_out", "iref_counts_out", "istatus", "isrc_rows", "isrc_lens",
          "icu_q_lens", "ipage_map", "inum_live")


def _pages_args(where: str, block_table, seq_lens, ref_counts, table_out, lens_out, refs_out, status, src_rows=None, src_lens=None, cu_q_lens=None,
                page_map=None, num_live=None):
    """(struct without the data, index of the GPU); an output that is None is its input."""
    (index, table, _, lens, nlens, refs, num_blocks, to, nto, lens_to, nlens_to, refs_to, nrefs, st, nst, src, rows, cut, ncut, cu, ncu, pm, npm, live,
     nlive) = _look(where, block_table, _PAGES, block_table, seq_lens, ref_counts, block_table if table_out is None else table_out,
                    seq_lens if lens_out is None else lens_out, ref_counts if refs_out is None else refs_out, status, src_rows, src_lens, cu_q_lens,
                    page_map, num_live)
    if block_table.dim() != 2:
        raise HookError(2, f"{where} (block_table: shape)")
    num_seqs, max_blocks = block_table.shape
    new_rows = num_seqs if src_rows is None else rows
    if table_out is not None and (table_out.dim() != 2 or table_out.shape[1] != max_blocks):
        raise HookError(2, f"{where} (block_table_out: shape)")
    if (nlens != num_seqs or nst != 1 or nrefs != num_blocks or nto != new_rows * max_blocks or nlens_to != new_rows or
            (src_lens is not None and ncut != rows) or (cu_q_lens is not None and ncu != num_seqs + 1) or
            (page_map is not None and (npm != num_blocks or nlive != 1))):
        raise HookError(2, f"{where} (shape)")
    if (num_seqs | max_blocks | num_blocks | rows) > _INT32_MAX:
        raise HookError(3, f"{where} (sizes)")
    return HookPagesArgs(num_seqs, max_blocks, num_blocks, 16, table, lens, refs, to, lens_to, refs_to, st, rows, src, cut, cu, pm, live), index


_CACHES: dict = {}      # by the length of a list of caches: what _look is to look for in them and in the scratch


def _pages_data(where: str, a, caches, like, workspace, index: int, stream):
    """Fills in the caches (a list of [num_blocks, Hkv, 16, d] tensors, or one tensor of them stacked) and the scratch; returns
    what has to live until the call has returned."""
    stacked = isinstance(caches, torch.Tensor)
    each = (caches,) if stacked else tuple(caches)
    n = len(each)
    spec = _CACHES.get(n)
    if spec is None:
        spec = _CACHES[n] = tuple(f"ccaches[{i}]" for i in range(n)) + ("cworkspace",)
    if workspace is None:
        with _taken_on(stream, index):
            workspace = torch.empty(pages_workspace_bytes(a.num_seqs, a.num_blocks), dtype=torch.uint8, device=index)
    seen = _look(where, like, spec, *each, workspace)
    a.workspace, a.workspace_bytes = seen[-2], workspace.numel() * workspace.element_size()
    pointers = seen[1:-2:2]
    if n:
        shape, dtype = seen[2], each[0].dtype
        if len(shape) != (5 if stacked else 4) or shape[-4] != a.num_blocks or shape[-2] != 16:
            raise HookError(2, f"{where} (caches: shape)")
        if n > 1 and any(s != shape for s in seen[4:-2:2]) or any(c.dtype is not dtype for c in each):
            raise HookError(2, f"{where} (caches: shape, dtype)")
        if shape[-3] > _INT32_MAX:
            raise HookError(3, f"{where} (caches: sizes)")
        a.num_kv_heads, a.row_bytes = shape[-3], shape[-1] * each[0].element_size()
        if stacked:
            n, step = shape[0], shape[1] * shape[2] * 16 * a.row_bytes
            pointers = range(pointers[0], pointers[0] + n * step, step) if n and step else ()
    array = (ctypes.c_void_p * (n or 1))(*pointers)
    a.num_caches, a.caches = n, array
    return array, workspace


@functools.lru_cache(maxsize=64)
def pages_workspace_bytes(num_seqs: int, num_blocks: int) -> int:
    """Scratch bytes of ``hook_pages_append`` and ``hook_pages_compact``."""
    a = HookPagesArgs()
    a.num_seqs, a.num_blocks = num_seqs, num_blocks
    return int(load_library().hook_pages_workspace_bytes(a))


def hook_pages_fork(src_rows, block_table, seq_lens, ref_counts, block_table_out, seq_lens_out, status, src_lens=None,
                    ref_counts_out=None, stream=None):
    """Replaces a block table by block_table_out / seq_lens_out, whose row j takes the first src_lens[j] (None: all) tokens of row
    src_rows[j], or is empty where that is -1; reference counts follow (in place unless ref_counts_out is given).  Bits of PAGES_* are
    added to `status`."""
    where = "hook_pages_fork"
    if src_rows is None or block_table_out is None or seq_lens_out is None:      # (a table of no rows is empty tensors)
        raise HookError(1, "hook_pages_fork (src_rows, block_table_out, seq_lens_out)")
    a, index = _pages_args(where, block_table, seq_lens, ref_counts, block_table_out, seq_lens_out, ref_counts_out, status, src_rows, src_lens)
    _launch((_lib or load_library()).hook_pages_fork, a, index, stream, where)


def hook_pages_append(cu_q_lens, block_table, seq_lens, ref_counts, caches, status, block_table_out=None, seq_lens_out=None,
                      ref_counts_out=None, workspace=None, stream=None):
    """Room for the new tokens of each row: lengths grow, pages are taken, last pages that others hold too are copied in every
    cache.  In place unless outputs are given; all or nothing (PAGES_FULL in `status`)."""
    where = "hook_pages_append"
    a, index = _pages_args(where, block_table, seq_lens, ref_counts, block_table_out, seq_lens_out, ref_counts_out, status, cu_q_lens=cu_q_lens)
    keep = _pages_data(where, a, caches, block_table, workspace, index, stream)
    _launch((_lib or load_library()).hook_pages_append, a, index, stream, where)
    del keep


def hook_pages_compact(block_table, seq_lens, ref_counts, caches, page_map, num_live, status, block_table_out=None,
                       ref_counts_out=None, workspace=None, stream=None):
    """Moves the live pages to the front of every cache and renumbers the table and the counts (in place unless outputs are
    given); page_map receives every page's new number (-1: free), num_live how many there are."""
    where = "hook_pages_compact"
    a, index = _pages_args(where, block_table, seq_lens, ref_counts, block_table_out, None, ref_counts_out, status, page_map=page_map, num_live=num_live)
    keep = _pages_data(where, a, caches, block_table, workspace, index, stream)
    _launch((_lib or load_library()).hook_pages_compact, a, index, stream, where)
    del keep


_LOGITS = ("rlogits", "rout", "ihistory", "icu_history", "iprompt_lens", "frepetition", "ffrequency", "fpresence", "icu_bias", "ibias_ids",
           "fbias_values", "imask", "imask_rows")


def hook_steer_logits(logits, out=None, history=None, cu_history=None, prompt_lens=None, repetition=None, frequency=None,
                      presence=None, cu_bias=None, bias_ids=None, bias_values=None, mask=None, mask_rows=None, stream=None):
    """Penalties for repeated tokens, a bias list and a grammar mask (int32 words, a set bit allows its token) on logits [rows, vocab], in
    place unless `out` is given.  Lists are int32 with prefix sums cu_*.  Returns the result."""
    where = "hook_steer_logits"
    if out is None:
        out = logits
    (index, x, xs, xn, y, ys, yn, h, nh, cuh, ncuh, pl, npl, rep, nrep, fr, nfr, pr, npr, cub, ncub, bi, nbi, bv, nbv, m, nm, mr,
     nmr) = _look(where, logits, _LOGITS, logits, out, history, cu_history, prompt_lens, repetition, frequency, presence, cu_bias, bias_ids,
                  bias_values, mask, mask_rows)
    dt = logits.dtype
    if dt not in _DT or len(xn) != 2:
        raise HookError(3, "hook_steer_logits (dtype)")
    rows, vocab = xn
    words = (vocab + 31) // 32
    if (yn != xn or (cu_history is not None and ncuh != rows + 1) or (prompt_lens is not None and npl != rows) or (repetition is not None and nrep != rows) or
            (frequency is not None and nfr != rows) or (presence is not None and npr != rows) or (cu_bias is not None and ncub != rows + 1) or nbi != nbv or
            (mask_rows is not None and nmr != rows) or (mask is not None and (mask.dim() != 2 or mask.shape[1] != words))):
        raise HookError(2, "hook_steer_logits (shape)")
    masks = nm // words if words else 0
    if (rows | vocab | nh | nbi | masks) > _INT32_MAX:
        raise HookError(3, "hook_steer_logits (sizes)")
    a = HookSteerLogitsArgs(rows, vocab, _DT[dt], x, y, xs, ys, nh, h, cuh, pl, rep, fr, pr, nbi, cub, bi, bv, masks, m, mr)
    _launch((_lib or load_library()).hook_steer_logits, a, index, stream, where)
    return out
