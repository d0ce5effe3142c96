"""Thin ctypes binding of the C ABI in include/asr.h (argument marshalling only).

Every computation runs in the HIP library; this module only converts Python
values and torch/numpy buffers to pointers.  Importing it raises if the
library has not been built (python -m paper_2603_11273_amd.build).
"""
from __future__ import annotations

import ctypes as C
import os
import threading

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libasr_mi355x.so")

ASR_OK, ASR_EINVAL, ASR_ENOMEM, ASR_EFULL, ASR_ENOTFOUND, ASR_ESTATE, ASR_ENODEV, ASR_EDEVICE = range(8)
NOT_WRITTEN = -(1 << 31)     # in a result before a call: no token, no policy
STATUS_NAMES = ["OK", "EINVAL", "ENOMEM", "EFULL", "ENOTFOUND", "ESTATE", "ENODEV", "EDEVICE"]
FCFS, SJF, HRRN = 0, 1, 2
F32, BF16 = 0, 1
(K_MEL, K_GEMM, K_ATTN, K_LN, K_DGEMM, K_DATTN, K_VOCAB, K_OTHER, K_PREFILL, K_DECODE,
 K_ENCODE, K_XKV) = range(12)
KERNEL_CLASSES = ["mel", "gemm", "attn", "ln", "dgemm", "dattn", "vocab", "other", "prefill",
                  "decode", "encode", "xkv"]
TIME_ALL = (1 << len(KERNEL_CLASSES)) - 1

EXPORTED = [
    "asr_create", "asr_destroy", "asr_last_error", "asr_workspace_size", "asr_bind",
    "asr_n_params", "asr_param_numel", "asr_load_weights", "asr_set_policy", "asr_submit",
    "asr_rank", "asr_pop_batch", "asr_queue_len", "asr_step", "asr_release_slot",
    "asr_slot_info", "asr_set_encoder_streams", "asr_set_decode_graphs", "asr_set_timing",
    "asr_get_timing",
    "asr_reset_timing",
    "asr_debug_logmel", "asr_debug_encode", "asr_debug_attention", "asr_debug_set_encoder_out",
    "asr_debug_get_kv",
    "asr_debug_set_self_kv", "asr_logmel_noalloc", "asr_serve_config", "asr_serve_step",
    "asr_serve_plan",
    "asr_serve_tokens", "asr_serve_simulate", "asr_serve_stats",
    "asr_attend_shared_size", "asr_attend_shared", "asr_logit_rules_size", "asr_logit_rules",
    "asr_write_pages", "asr_attend_pages_size", "asr_attend_pages", "asr_next_tables_size",
    "asr_next_tables", "asr_sample_size", "asr_sample",
    "asr_hypotheses_size", "asr_bind_hypotheses", "asr_fork_slot", "asr_set_masks",
    "asr_set_slot_rules", "asr_set_slot_mask", "asr_step_topk",
]


class ModelCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_mels", "d_model", "n_enc", "n_dec", "n_head", "d_ffn", "vocab", "dtype",
        "max_slots", "max_prefill", "max_decode", "max_queue")]


class StepIn(C.Structure):
    _fields_ = [("n_prefill", C.c_int32), ("prefill_ids", C.POINTER(C.c_int64)),
                ("n_decode", C.c_int32), ("slots", C.POINTER(C.c_int32)),
                ("tokens", C.POINTER(C.c_int32)), ("logits", C.POINTER(C.c_float))]


class StepOut(C.Structure):
    _fields_ = [("slot_of", C.POINTER(C.c_int32)), ("argmax", C.POINTER(C.c_int32)),
                ("done", C.POINTER(C.c_int32))]


class ServeCfg(C.Structure):
    _fields_ = [("kv_capacity", C.c_int64), ("cross_tokens", C.c_int32),
                ("max_admit", C.c_int32), ("tok_num", C.c_int32), ("tok_den", C.c_int32),
                ("start_token", C.c_int32), ("dynamic", C.c_int32), ("depth_low", C.c_int32),
                ("starve_num", C.c_int64), ("starve_den", C.c_int64), ("overlap", C.c_int32)]


class ServeOut(C.Structure):
    _fields_ = [("cap", C.c_int32), ("policy", C.c_int32),
                ("preempted", C.POINTER(C.c_int64)), ("n_preempted", C.c_int32),
                ("admitted", C.POINTER(C.c_int64)), ("admitted_slot", C.POINTER(C.c_int32)),
                ("n_admitted", C.c_int32),
                ("decoded", C.POINTER(C.c_int64)), ("token", C.POINTER(C.c_int32)),
                ("n_decoded", C.c_int32),
                ("finished", C.POINTER(C.c_int64)), ("n_finished", C.c_int32)]


class SimCost(C.Structure):
    _fields_ = [("prefill_us", C.c_int64), ("step_us", C.c_int64), ("row_us", C.c_int64)]


class Keys(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("slot_stride", C.c_int64),
                ("head_stride", C.c_int64), ("pos_stride", C.c_int64), ("slots", C.c_int32),
                ("positions", C.c_int32), ("slot", C.c_void_p), ("first", C.c_void_p),
                ("len", C.c_void_p)]


class Attention(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "dtype", "n_head", "n_kv_head", "rows", "groups", "max_group", "max_prefix", "max_own",
        "part_keys")] + [
        ("scale", C.c_float), ("q", C.c_void_p), ("q_ld", C.c_int64), ("out", C.c_void_p),
        ("out_ld", C.c_int64), ("group_start", C.c_void_p), ("row_of", C.c_void_p),
        ("prefix", Keys), ("own", Keys)]


class Rules(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "rows", "vocab", "sets", "masks", "k")] + [
        ("logits", C.c_void_p), ("ld", C.c_int64), ("set", C.c_void_p), ("history", C.c_void_p),
        ("history_ld", C.c_int64), ("history_len", C.c_void_p), ("prompt_len", C.c_void_p),
        ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p),
        ("bias_token", C.c_void_p), ("bias_value", C.c_void_p), ("bias_ld", C.c_int64),
        ("bias_len", C.c_void_p), ("mask", C.c_void_p), ("mask_ld", C.c_int64),
        ("mask_of", C.c_void_p), ("temperature", C.c_void_p), ("out", C.c_void_p),
        ("out_ld", C.c_int64), ("token", C.c_void_p), ("logprob", C.c_void_p)]


class Pages(C.Structure):
    _fields_ = [("kv_heads", C.c_int32), ("page", C.c_int32), ("pages", C.c_int32), ("codes", C.c_void_p),
                ("page_stride", C.c_int64), ("scales", C.c_void_p), ("scale_stride", C.c_int64),
                ("table", C.c_void_p), ("table_ld", C.c_int64), ("sequences", C.c_int32),
                ("columns", C.c_int32)]


class PageTokens(C.Structure):
    _fields_ = [("cache", Pages), ("dtype", C.c_int32), ("tokens", C.c_int32), ("max_new", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("ld", C.c_int64), ("token_start", C.c_void_p),
                ("length", C.c_void_p)]


class PageQueries(C.Structure):
    _fields_ = [("cache", Pages)] + [(n, C.c_int32) for n in (
        "dtype", "n_head", "rows", "max_rows", "max_keys", "part_keys")] + [
        ("scale", C.c_float), ("q", C.c_void_p), ("q_ld", C.c_int64), ("out", C.c_void_p),
        ("out_ld", C.c_int64), ("row_start", C.c_void_p), ("first", C.c_void_p), ("length", C.c_void_p)]


class NextTables(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("sequences", "columns", "page", "pages", "compact")] + [
        ("table", C.c_void_p), ("table_ld", C.c_int64), ("length", C.c_void_p), ("parent", C.c_void_p),
        ("want", C.c_void_p), ("new_table", C.c_void_p), ("new_ld", C.c_int64),
        ("new_length", C.c_void_p), ("room", C.c_void_p), ("info", C.c_void_p), ("codes", C.c_void_p),
        ("code_stride", C.c_int64), ("code_bytes", C.c_int64), ("scales", C.c_void_p),
        ("scale_stride", C.c_int64), ("scale_bytes", C.c_int64)]


class Sampling(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "rows", "vocab", "sets", "draws")] + [
        ("logits", C.c_void_p), ("ld", C.c_int64), ("u", C.c_void_p), ("set", C.c_void_p),
        ("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p),
        ("token", C.c_void_p), ("logprob", C.c_void_p), ("kept", C.c_void_p)]


class SlotRules(C.Structure):
    _fields_ = [("repetition", C.c_float), ("frequency", C.c_float), ("presence", C.c_float),
                ("temperature", C.c_float), ("n_prompt", C.c_int32), ("mask", C.c_int32),
                ("n_bias", C.c_int32), ("bias_token", C.POINTER(C.c_int32)),
                ("bias_value", C.POINTER(C.c_float))]


class AsrError(RuntimeError):
    """An error status.  `results`: what the call would have returned, where it did all its work and
    only a row of it has no next token (Context.step, Context.serve_step); None otherwise."""

    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 8 else status}: {msg}")
        self.status = status
        self.results = None


def _load():
    # torch bundles its own HIP runtime (soname libamdhip64.so.7).  Loading it
    # first makes the library bind to that same runtime by soname, so device
    # pointers and streams from torch are valid here; loading the library
    # first would pull a second HIP runtime into the process.
    try:
        import torch  # noqa: F401
    except Exception:  # pragma: no cover - queue-only use without torch
        pass
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2603_11273_amd.build`")
    lib = C.CDLL(LIB_PATH)
    P, i32, i64, f, vp = C.POINTER, C.c_int32, C.c_int64, C.c_float, C.c_void_p
    sig = {
        "asr_create": [P(ModelCfg), i32, P(vp)],
        "asr_destroy": [vp],
        "asr_last_error": [],
        "asr_workspace_size": [vp, P(C.c_size_t)],
        "asr_bind": [vp, vp, C.c_size_t, vp],
        "asr_n_params": [vp, P(i32)],
        "asr_param_numel": [vp, i32, P(i64)],
        "asr_load_weights": [vp, P(vp), i32, i32],
        "asr_set_policy": [vp, i32, i32, i32],
        "asr_submit": [vp, i64, vp, i64, i32, i64, i64, i32, i32],
        "asr_rank": [vp, i64, P(i64), i32, P(i32)],
        "asr_pop_batch": [vp, i64, i32, P(i64), P(i32)],
        "asr_queue_len": [vp, P(i32)],
        "asr_step": [vp, P(StepIn), P(StepOut)],
        "asr_release_slot": [vp, i32],
        "asr_slot_info": [vp, i32, P(i32), P(i64), P(i32), P(i32)],
        "asr_set_encoder_streams": [vp, i32],
        "asr_set_decode_graphs": [vp, i32],
        "asr_set_timing": [vp, i32],
        "asr_get_timing": [vp, i32, P(C.c_double), P(i64), P(C.c_double), P(C.c_double)],
        "asr_reset_timing": [vp],
        "asr_debug_logmel": [vp, P(vp), P(i64), i32, i32, P(f)],
        "asr_debug_encode": [vp, P(vp), P(i64), i32, i32, P(f)],
        "asr_debug_attention": [vp, P(f), P(f), P(f), i32, P(f)],
        "asr_debug_set_encoder_out": [vp, P(i32), P(i64), P(i32), i32, vp, i32],
        "asr_debug_get_kv": [vp, i32, i32, P(f)],
        "asr_debug_set_self_kv": [vp, i32, vp, i32, i32],
        "asr_logmel_noalloc": [P(vp), P(i64), i32, i32, vp, vp],
        "asr_serve_config": [vp, P(ServeCfg)],
        "asr_serve_step": [vp, i64, P(ServeOut)],
        "asr_serve_plan": [vp, i64, P(ServeOut)],
        "asr_serve_tokens": [vp, i64, P(i32), i32, P(i32)],
        "asr_serve_stats": [vp, P(i64)],
        "asr_serve_simulate": [vp, P(SimCost), i64, i32, P(i64), P(i64), P(i64), P(i32),
                               P(i32), P(i64), i64, P(i64)],
        "asr_attend_shared_size": [P(Attention), P(C.c_size_t)],
        "asr_attend_shared": [P(Attention), vp, C.c_size_t, vp],
        "asr_logit_rules_size": [P(Rules), P(C.c_size_t)],
        "asr_logit_rules": [P(Rules), vp, C.c_size_t, vp],
        "asr_write_pages": [P(PageTokens), vp],
        "asr_attend_pages_size": [P(PageQueries), P(C.c_size_t)],
        "asr_attend_pages": [P(PageQueries), vp, C.c_size_t, vp],
        "asr_next_tables_size": [P(NextTables), P(C.c_size_t)],
        "asr_next_tables": [P(NextTables), vp, C.c_size_t, vp],
        "asr_sample_size": [P(Sampling), P(C.c_size_t)],
        "asr_sample": [P(Sampling), vp, C.c_size_t, vp],
        "asr_hypotheses_size": [vp, i32, i32, P(C.c_size_t)],
        "asr_bind_hypotheses": [vp, i32, i32, vp, C.c_size_t],
        "asr_fork_slot": [vp, i32, i32],
        "asr_set_masks": [vp, i32, i32, vp],
        "asr_set_slot_rules": [vp, i32, P(SlotRules)],
        "asr_set_slot_mask": [vp, i32, i32],
        "asr_step_topk": [vp, P(StepIn), P(StepOut), i32, P(i32), P(f)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_char_p if name == "asr_last_error" else C.c_int
    return lib


lib = _load()


def _check(status, results=None):
    if status != ASR_OK:
        error = AsrError(status, lib.asr_last_error().decode())
        error.results = results
        raise error


def _ptr(a):
    """Address of a torch tensor or numpy array (contiguous)."""
    if a is None:
        return None
    if hasattr(a, "data_ptr"):
        assert a.is_contiguous()
        return a.data_ptr()
    assert a.flags["C_CONTIGUOUS"]
    return a.ctypes.data


def _i64(a):
    a = np.ascontiguousarray(a, dtype=np.int64)
    return a, a.ctypes.data_as(C.POINTER(C.c_int64))


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


def logmel_noalloc(clips, n_mels, out, stream=None):
    """asr_logmel_noalloc: normalised log-mel features of device clips (torch
    tensors, float32) into the device tensor out [n][3000][n_mels], on
    `stream` (torch.cuda.Stream; default: torch's current stream)."""
    import torch
    n = len(clips)
    for x in clips:
        if not (x.is_cuda and x.dtype == torch.float32):
            raise TypeError("clips must be float32 device tensors")
    if not (out.is_cuda and out.dtype == torch.float32 and tuple(out.shape) == (n, 3000, n_mels)):
        raise TypeError(f"out must be a float32 device tensor of shape ({n}, 3000, {n_mels})")
    ptrs = (C.c_void_p * n)(*[_ptr(x) for x in clips])
    ns = np.array([x.numel() for x in clips], np.int64)
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib.asr_logmel_noalloc(ptrs, ns.ctypes.data_as(C.POINTER(C.c_int64)), n, n_mels,
                                  _ptr(out), st))


class _Operator:
    """What the plans of the stateless operators share: the tensors they keep, their scratch and
    the call.  Tensors are taken as they lie (no copies) and must stay where they are; what is in
    them may change between calls.  A workspace given to a plan starts as zeros; plans may share
    one if their calls never overlap.  A plan's own may be used on any stream as soon as the plan is
    made (under capture: in that graph alone), and stays until the calls are done; calls held by a
    captured graph need the plan kept.

    A plan is for one call at a time.  Threads that call one take turns; calls on several streams,
    which share its scratch, are ordered by the program, or made through a plan for each stream."""

    def __init__(self, device, workspace, size, run, args):
        import torch
        if workspace is not None and (workspace.device != device or workspace.dtype != torch.uint8
                                      or not workspace.is_contiguous()):
            raise TypeError(f"workspace must be contiguous bytes (torch.uint8) on {device}")
        self._dev, self._run, self._args = device, run, args
        self._turn = threading.Lock()          # from a call's pointers in args to the library's return
        # the current stream's handle without a Stream object around it (1.8 us of a 10-us call)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda i: torch.cuda.current_stream(i).cuda_stream)
        self._ref = C.byref(args)
        n = C.c_size_t()
        _check(size(self._ref, C.byref(n)))
        self.workspace_bytes = n.value
        self._ws = workspace
        self._streams = None                   # a given block: its streams are the program's matter
        if workspace is None:
            self._ws = torch.zeros(max(n.value, 1), dtype=torch.uint8, device=device)
            # calls may come on any stream, and count on the zeros
            home = torch.cuda.current_stream(device)
            if not torch.cuda.is_current_stream_capturing():
                home.synchronize()
            self._streams = {home.cuda_stream}
        self._ws_ptr, self._ws_bytes = self._ws.data_ptr(), self._ws.numel()

    def _need(self, t, name, dtype, shape, device, ld=False):
        """A tensor's checks (contiguous; with ld, rows that are); its address."""
        if t is None:
            return None
        if t.dtype != dtype or t.shape != shape or t.device != device:
            raise TypeError(f"{name} must be {dtype} of shape {tuple(shape)} on {device}")
        if not (t.is_contiguous() or (ld and t.stride(-1) == 1)):
            raise TypeError(f"{name} must be contiguous")
        return t.data_ptr()

    @staticmethod
    def _ld(t):
        """Elements from row to row (of a single row torch may say anything)."""
        return t.stride(0) if t.shape[0] > 1 else t.shape[1]

    def _launch(self, stream):
        import torch
        st = self._raw_stream(self._dev.index) if stream is None else stream.cuda_stream
        if self._streams is not None and st not in self._streams:
            # the plan's own block is not to be handed out again before this stream is done with it
            self._ws.record_stream(torch.cuda.current_stream(self._dev) if stream is None else stream)
            self._streams.add(st)
        if torch.cuda.current_device() == self._dev.index:
            e = self._run(self._ref, self._ws_ptr, self._ws_bytes, st)
            if e:
                _check(e)
            return
        with torch.cuda.device(self._dev):
            _check(self._run(self._ref, self._ws_ptr, self._ws_bytes, st))


class SharedAttention(_Operator):
    """asr_attend_shared as a plan: caches, groups and lengths once, then plan(q, out) per step.

    prefix_k, prefix_v, own_k, own_v: [slots][kv heads][positions][64] views of a cache (float32
    or bfloat16, the dims of a head contiguous, k and v with the same strides).  Group g holds rows
    row_of[group_start[g] : group_start[g + 1]] (row_of None: the rows themselves), at most
    max_group of them.  The int32 device tensors group_start [groups + 1], row_of [rows],
    prefix_slot / prefix_first / prefix_len [groups] and own_slot / own_first / own_len [rows] are
    read at every call.  max_prefix, max_own bound the lengths (default: the positions).
    plan(q, out): q float32 [rows][n_head * 64], out [rows][n_head * 64] in the cache's type, on
    `stream` (default: torch's current stream).  One call at a time: calls that may overlap on the
    GPU need plans with a workspace each (default: one of the plan's own)."""

    def __init__(self, prefix_k=None, prefix_v=None, own_k=None, own_v=None, *, n_head, rows,
                 groups, max_group, group_start, row_of=None, prefix_slot=None, prefix_first=None,
                 prefix_len=None, max_prefix=None, own_slot=None, own_first=None, own_len=None,
                 max_own=None, scale=0.125, part_keys=0, workspace=None):
        import torch
        some = prefix_k if prefix_k is not None else own_k
        if some is None or some.dtype not in (torch.float32, torch.bfloat16) or not some.is_cuda:
            raise TypeError("caches must be float32 or bfloat16 device tensors")
        dev, i32 = some.device, torch.int32
        self._dtype = some.dtype

        def keys(k, v, slot, first, length, entries, name):
            if k is None:
                return Keys()
            if v is None or k.dim() != 4 or k.shape != v.shape or k.shape[3] != 64 or k.shape[1] != some.shape[1]:
                raise TypeError(f"{name}: k and v must be [slots][kv heads][positions][64]")
            if any(t.device != dev or t.dtype != some.dtype for t in (k, v)):
                raise TypeError(f"{name}: k and v must be {some.dtype} on {dev}")
            # (of a dimension of one element torch may say anything)
            step, v_step = ([t.stride(i) if t.shape[i] > 1 else one for i, one in enumerate((0, 0, 64, 1))]
                            for t in (k, v))
            if step != v_step or step[3] != 1:
                raise TypeError(f"{name}: k and v must have the same strides, dims contiguous")
            idx = [self._need(t, f"{name}_{n}", i32, (entries,), dev)
                   for t, n in ((slot, "slot"), (first, "first"), (length, "len"))]
            return Keys(k.data_ptr(), v.data_ptr(), *step[:3], k.shape[0], k.shape[2], *idx)

        self._keep = (prefix_k, prefix_v, own_k, own_v, group_start, row_of, prefix_slot,
                      prefix_first, prefix_len, own_slot, own_first, own_len)
        most = [0 if k is None else k.shape[2] if m is None else m
                for k, m in ((prefix_k, max_prefix), (own_k, max_own))]
        args = Attention(
            BF16 if some.dtype == torch.bfloat16 else F32, n_head, some.shape[1], rows, groups,
            max_group, most[0], most[1], part_keys, scale, None, 0, None, 0,
            self._need(group_start, "group_start", i32, (groups + 1,), dev),
            self._need(row_of, "row_of", i32, (rows,), dev),
            keys(prefix_k, prefix_v, prefix_slot, prefix_first, prefix_len, groups, "prefix"),
            keys(own_k, own_v, own_slot, own_first, own_len, rows, "own"))
        self._shape = (rows, n_head * 64)
        super().__init__(dev, workspace, lib.asr_attend_shared_size, lib.asr_attend_shared, args)

    def __call__(self, q, out, stream=None):
        import torch
        a = self._args
        with self._turn:
            a.q = self._need(q, "q", torch.float32, self._shape, self._dev, ld=True)
            a.out = self._need(out, "out", self._dtype, self._shape, self._dev, ld=True)
            a.q_ld, a.out_ld = self._ld(q), self._ld(out)
            self._launch(stream)
        return out


class LogitRules(_Operator):
    """asr_logit_rules as a plan: rule sets once, then plan(logits, ...) per step.

    Row r follows rule set set[r] (None: r).  Device tensors, read at every call: set int32 [rows];
    history int32 [sets][n] with history_len and prompt_len int32 [sets]; repetition, frequency,
    presence, temperature float32 [sets]; bias_token int32 and bias_value float32 [sets][n] with
    bias_len int32 [sets]; mask int32 [masks][words] (bit v % 32 of word v / 32 set = allowed) with
    mask_of int32 [sets].  plan(logits, out, token, logprob): logits [rows][vocab] of `dtype`
    (float32 or bfloat16), out float32 [rows][vocab] or None (may be the logits themselves), token
    int32 and logprob float32 [rows][k].  One call at a time: calls that may overlap on the GPU
    need plans with a workspace each (default: one of the plan's own)."""

    def __init__(self, rows, vocab, dtype, *, k=0, sets=None, set=None, history=None,
                 history_len=None, prompt_len=None, repetition=None, frequency=None,
                 presence=None, bias_token=None, bias_value=None, bias_len=None, mask=None,
                 mask_of=None, temperature=None, device=None, workspace=None):
        import torch
        i32, f32 = torch.int32, torch.float32
        if dtype not in (f32, torch.bfloat16):
            raise TypeError("logits must be float32 or bfloat16")
        given = [t for t in (set, history, repetition, frequency, presence, bias_token, mask,
                             temperature) if t is not None]
        dev = torch.device(device if device is not None else
                           given[0].device if given else torch.cuda.current_device())
        if dev.type != "cuda":
            raise TypeError(f"rules are applied on a GPU, not on {dev}")
        if dev.index is None:
            dev = torch.device(dev.type, torch.cuda.current_device())
        n = rows if sets is None else sets
        need = self._need
        self._keep = (set, history, history_len, prompt_len, repetition, frequency, presence,
                      bias_token, bias_value, bias_len, mask, mask_of, temperature)
        hist_n = 0 if history is None else history.shape[-1]
        bias_n = 0 if bias_token is None else bias_token.shape[-1]
        masks, words = (0, 0) if mask is None else mask.shape
        one = lambda t, name, kind: need(t, name, kind, (n,), dev)  # noqa: E731
        args = Rules(
            BF16 if dtype == torch.bfloat16 else F32, rows, vocab, n, masks, k, None, 0,
            need(set, "set", i32, (rows,), dev), need(history, "history", i32, (n, hist_n), dev),
            hist_n, one(history_len, "history_len", i32), one(prompt_len, "prompt_len", i32),
            one(repetition, "repetition", f32), one(frequency, "frequency", f32),
            one(presence, "presence", f32), need(bias_token, "bias_token", i32, (n, bias_n), dev),
            need(bias_value, "bias_value", f32, (n, bias_n), dev), bias_n,
            one(bias_len, "bias_len", i32), need(mask, "mask", i32, (masks, words), dev), words,
            one(mask_of, "mask_of", i32), one(temperature, "temperature", f32), None, 0, None, None)
        self._dtype, self._shape, self._best = dtype, (rows, vocab), (rows, k)
        super().__init__(dev, workspace, lib.asr_logit_rules_size, lib.asr_logit_rules, args)

    def __call__(self, logits, out=None, token=None, logprob=None, stream=None):
        import torch
        a = self._args
        with self._turn:
            a.logits = self._need(logits, "logits", self._dtype, self._shape, self._dev, ld=True)
            a.ld = self._ld(logits)
            a.out = self._need(out, "out", torch.float32, self._shape, self._dev, ld=True)
            a.out_ld = 0 if out is None else self._ld(out)
            a.token = self._need(token, "token", torch.int32, self._best, self._dev)
            a.logprob = self._need(logprob, "logprob", torch.float32, self._best, self._dev)
            self._launch(stream)


def _no_scratch(args, bytes):
    """The _size call of an operator without scratch."""
    return ASR_OK


class _Paged(_Operator):
    """What the plans over a pool of pages share: the pool and its tables.

    codes uint8 [pages][2][kv heads][page / 64][64][64] and scales float32
    [pages][2][kv heads][page / 64], on the GPU, everything inside a page contiguous (pages may
    lie further apart: codes[:, layer] of a pool of several layers); keys [position][dim] in a
    block, values [dim][position].  table int32 [sequences][columns]."""

    def _pages(self, codes, scales, table):
        import torch
        if not (codes.is_cuda and codes.dtype in (torch.uint8, torch.float8_e4m3fn) and codes.dim() == 6
                and codes.shape[1] == 2 and tuple(codes.shape[4:]) == (64, 64)):
            raise TypeError("codes must be device bytes of shape [pages][2][kv heads][page / 64][64][64]")
        dev, n = codes.device, codes.shape[0]
        if scales.device != dev or scales.dtype != torch.float32 or scales.shape != codes.shape[:4]:
            raise TypeError(f"scales must be float32 of shape {tuple(codes.shape[:4])} on {dev}")
        if n and not (codes[0].is_contiguous() and scales[0].is_contiguous()):
            raise TypeError("codes and scales must be contiguous inside a page")
        if table.dim() != 2:
            raise TypeError("table must be [sequences][columns]")
        self._need(table, "table", torch.int32, table.shape, dev, ld=True)
        stride = codes.stride(0) if n > 1 else max(codes[0].numel() if n else 0, 0)
        scale_stride = scales.stride(0) if n > 1 else scales[0].numel() if n else 0
        self._keep = [codes, scales, table]
        return dev, Pages(codes.shape[2], codes.shape[3] * 64, n, codes.data_ptr(), stride,
                          scales.data_ptr(), scale_stride, table.data_ptr(), self._ld(table),
                          table.shape[0], table.shape[1])


class PageWrite(_Paged):
    """asr_write_pages as a plan: pool, tables and lengths once, then plan(k, v) per step.

    codes, scales, table: a pool of pages (see _Paged).  Sequence s holds length[s] positions
    and gets tokens token_start[s] .. token_start[s + 1] - 1 behind them (None: token s alone), at
    most max_new.  The int32 device tensors table, length [sequences] and token_start
    [sequences + 1] are read at every call.  plan(k, v): [tokens][kv heads * 64] of `dtype`
    (float32 or bfloat16), rows the same distance apart, on `stream` (default: torch's current
    stream)."""

    def __init__(self, codes, scales, table, length, *, tokens, dtype, token_start=None, max_new=1):
        import torch
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("keys and values must be float32 or bfloat16")
        dev, pages = self._pages(codes, scales, table)
        n = table.shape[0]
        args = PageTokens(pages, BF16 if dtype == torch.bfloat16 else F32, tokens, max_new, None, None, 0,
                          self._need(token_start, "token_start", torch.int32, (n + 1,), dev),
                          self._need(length, "length", torch.int32, (n,), dev))
        if length is None:
            raise TypeError("length must be given")
        self._keep += [length, token_start]
        self._dtype, self._shape = dtype, (tokens, codes.shape[2] * 64)
        run = lambda ref, ws, n, stream: lib.asr_write_pages(ref, stream)  # noqa: E731
        super().__init__(dev, torch.empty(0, dtype=torch.uint8, device=dev), _no_scratch, run, args)

    def __call__(self, k, v, stream=None):
        a = self._args
        with self._turn:
            a.k = self._need(k, "k", self._dtype, self._shape, self._dev, ld=True)
            a.v = self._need(v, "v", self._dtype, self._shape, self._dev, ld=True)
            if a.k is None or a.v is None or self._ld(k) != self._ld(v):
                raise TypeError("k and v must be given, their rows the same distance apart")
            a.ld = self._ld(k)
            self._launch(stream)


class PagedAttention(_Paged):
    """asr_attend_pages as a plan: pool, tables and rows once, then plan(q, out) per step.

    codes, scales, table: a pool of pages (see _Paged).  Rows row_start[s] .. row_start[s + 1] - 1
    are of sequence s (None: row s alone), at most max_rows of them; row r attends to positions
    first[r] (None: 0) .. length[r] - 1.  The int32 device tensors table, row_start
    [sequences + 1], first and length [rows] are read at every call.  max_keys bounds the lengths
    (default: what the table holds).  plan(q, out): q float32 [rows][n_head * 64], out
    [rows][n_head * 64] of `dtype` (float32 or bfloat16), on `stream` (default: torch's current
    stream).  One call at a time: calls that may overlap on the GPU need plans with a workspace
    each (default: one of the plan's own)."""

    def __init__(self, codes, scales, table, length, *, n_head, rows, row_start=None, max_rows=1,
                 first=None, max_keys=None, scale=0.125, dtype=None, part_keys=0, workspace=None):
        import torch
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("out must be float32 or bfloat16")
        dev, pages = self._pages(codes, scales, table)
        if length is None:
            raise TypeError("length must be given")
        one = lambda t, name, n: self._need(t, name, torch.int32, (n,), dev)  # noqa: E731
        most = min(pages.columns * pages.page, (1 << 31) - 1) if max_keys is None else max_keys
        args = PageQueries(pages, BF16 if dtype == torch.bfloat16 else F32, n_head, rows, max_rows, most,
                           part_keys, scale, None, 0, None, 0, one(row_start, "row_start", pages.sequences + 1),
                           one(first, "first", rows), one(length, "length", rows))
        self._keep += [length, row_start, first]
        self._dtype, self._shape = dtype, (rows, n_head * 64)
        super().__init__(dev, workspace, lib.asr_attend_pages_size, lib.asr_attend_pages, args)

    def __call__(self, q, out, stream=None):
        import torch
        a = self._args
        with self._turn:
            a.q = self._need(q, "q", torch.float32, self._shape, self._dev, ld=True)
            a.out = self._need(out, "out", self._dtype, self._shape, self._dev, ld=True)
            if a.q is None or a.out is None:
                raise TypeError("q and out must be given")
            a.q_ld, a.out_ld = self._ld(q), self._ld(out)
            self._launch(stream)
        return out


class PageTables(_Operator):
    """asr_next_tables as a plan: the tables of a next step from those of this one.

    codes and scales: a pool, pages first, everything inside a page contiguous (all layers of a
    model in a page, or one), or None (the program copies its data itself; then pages and page say what
    the pool is).  table int32 [sequences][columns] and length [sequences] are those before the call;
    new_table and new_length those after it, or None: in place.  parent [sequences]: the
    sequence that each goes on from (None: itself; outside the range: none); want: the positions
    that each must have room for.  room [sequences] and info [4] (pages in use, missing, copied,
    moved) may be None.  Device tensors of int32, read at every call.  plan(compact=False): with
    compact the pages in use end up as the first of the pool.  One call at a time: calls that may
    overlap on the GPU need plans with a workspace each (default: one of the plan's own)."""

    def __init__(self, codes, scales, table, length, *, parent=None, want=None, new_table=None,
                 new_length=None, room=None, info=None, page=None, pages=None, workspace=None):
        import torch
        i32 = torch.int32
        if table is None or not table.is_cuda or table.dim() != 2 or length is None:
            raise TypeError("table must be a device tensor of [sequences][columns], with its lengths")
        dev, (n, columns) = table.device, table.shape
        if codes is not None:
            if codes.dim() < 3 or codes.dtype not in (torch.uint8, torch.float8_e4m3fn):
                raise TypeError("codes must be bytes, pages first")
            page = codes.shape[-3] * 64 if page is None else page
            pages = codes.shape[0] if pages is None else pages
        if page is None or pages is None:
            raise TypeError("without codes, page and pages must be given")

        def pool(t, name):
            if t is None:
                return None, 0, 0
            if t.device != dev or t.shape[0] < pages or (pages and not t[0].is_contiguous()):
                raise TypeError(f"{name} must be {pages} pages on {dev}, contiguous inside a page")
            size = t[0].numel() * t.element_size() if pages else 0
            return t.data_ptr(), t.stride(0) * t.element_size() if pages > 1 else size, size

        new_table = table if new_table is None else new_table
        new_length = length if new_length is None else new_length
        one = lambda t, name: self._need(t, name, i32, (n,), dev)  # noqa: E731
        args = NextTables(n, columns, page, pages, 0, self._need(table, "table", i32, (n, columns), dev, ld=True),
                          self._ld(table), one(length, "length"), one(parent, "parent"), one(want, "want"),
                          self._need(new_table, "new_table", i32, (n, columns), dev, ld=True),
                          self._ld(new_table), one(new_length, "new_length"), one(room, "room"),
                          self._need(info, "info", i32, (4,), dev), *pool(codes, "codes"), *pool(scales, "scales"))
        self._keep = (codes, scales, table, length, parent, want, new_table, new_length, room, info)
        super().__init__(dev, workspace, lib.asr_next_tables_size, lib.asr_next_tables, args)

    def __call__(self, compact=False, stream=None):
        with self._turn:
            self._args.compact = int(bool(compact))
            self._launch(stream)


class Sampler(_Operator):
    """asr_sample as a plan: parameter sets once, then plan(logits, u, token, ...) per step.

    Row r follows parameter set set[r] (None: r).  Device tensors, read at every call: set int32
    [rows]; temperature, top_p, min_p float32 and top_k int32 [sets].  plan(logits, u, token,
    logprob, kept): logits [rows][vocab] of `dtype` (float32 or bfloat16), u float32
    [rows][draws] in [0, 1), token int32 and logprob float32 [rows][draws], kept int32 [rows]
    (logprob and kept may be None).  The call has no scratch, so calls of one plan may overlap on
    the GPU where their outputs lie apart; a workspace that is given is left as it is."""

    def __init__(self, rows, vocab, dtype, *, draws=1, sets=None, set=None, temperature=None, top_k=None,
                 top_p=None, min_p=None, device=None, workspace=None):
        import torch
        i32, f32 = torch.int32, torch.float32
        if dtype not in (f32, torch.bfloat16):
            raise TypeError("logits must be float32 or bfloat16")
        given = [t for t in (set, temperature, top_k, top_p, min_p) if t is not None]
        dev = torch.device(device if device is not None else
                           given[0].device if given else torch.cuda.current_device())
        if dev.type != "cuda":
            raise TypeError(f"tokens are drawn on a GPU, not on {dev}")
        if dev.index is None:
            dev = torch.device(dev.type, torch.cuda.current_device())
        n = rows if sets is None else sets
        one = lambda t, name, kind: self._need(t, name, kind, (n,), dev)  # noqa: E731
        args = Sampling(BF16 if dtype == torch.bfloat16 else F32, rows, vocab, n, draws, None, 0, None,
                        self._need(set, "set", i32, (rows,), dev), one(temperature, "temperature", f32),
                        one(top_k, "top_k", i32), one(top_p, "top_p", f32), one(min_p, "min_p", f32),
                        None, None, None)
        self._keep = (set, temperature, top_k, top_p, min_p)
        self._dtype, self._shape, self._drawn = dtype, (rows, vocab), (rows, draws)
        super().__init__(dev, workspace, lib.asr_sample_size, lib.asr_sample, args)

    def __call__(self, logits, u, token, logprob=None, kept=None, stream=None):
        import torch
        a = self._args
        with self._turn:
            a.logits = self._need(logits, "logits", self._dtype, self._shape, self._dev, ld=True)
            a.ld = self._ld(logits)
            a.u = self._need(u, "u", torch.float32, self._drawn, self._dev)
            a.token = self._need(token, "token", torch.int32, self._drawn, self._dev)
            a.logprob = self._need(logprob, "logprob", torch.float32, self._drawn, self._dev)
            a.kept = self._need(kept, "kept", torch.int32, self._shape[:1], self._dev)
            self._launch(stream)


def model_cfg(shape, max_slots=8, max_prefill=1, max_decode=8, max_queue=4096) -> ModelCfg:
    """asr_model_cfg from a synth.ModelShape (or anything with the same fields)."""
    return ModelCfg(shape.n_mels, shape.d_model, shape.n_enc, shape.n_dec, shape.n_head,
                    shape.d_ffn, shape.vocab, BF16 if shape.dtype == "bf16" else F32,
                    max_slots, max_prefill, max_decode, max_queue)


class Context:
    """One asr_ctx.  device=-1 gives a queue-only context (no GPU calls)."""

    def __init__(self, cfg: ModelCfg, device: int = 0):
        self.cfg = cfg
        self.device = device
        h = C.c_void_p()
        _check(lib.asr_create(C.byref(cfg), device, C.byref(h)))
        self.h = h
        self._block = None
        self._keep = []
        self._serve_cap = max(cfg.max_slots, 1)

    def close(self):
        if self.h:
            lib.asr_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- memory ---------------------------------------------------------------
    def workspace_size(self) -> int:
        n = C.c_size_t()
        _check(lib.asr_workspace_size(self.h, C.byref(n)))
        return n.value

    def bind(self, block=None, stream=None):
        """Binds a device block (torch uint8 tensor; allocated here when None)."""
        import torch
        if block is None:
            block = torch.empty(self.workspace_size(), dtype=torch.uint8,
                                device=f"cuda:{self.device}")
        if stream is None:
            stream = torch.cuda.current_stream(self.device).cuda_stream
        _check(lib.asr_bind(self.h, C.c_void_p(block.data_ptr()), block.numel(),
                            C.c_void_p(stream)))
        self._block = block
        return block

    def n_params(self) -> int:
        n = C.c_int32()
        _check(lib.asr_n_params(self.h, C.byref(n)))
        return n.value

    def param_numel(self, i) -> int:
        n = C.c_int64()
        _check(lib.asr_param_numel(self.h, i, C.byref(n)))
        return n.value

    def load_weights(self, tensors, on_device: bool):
        arr = (C.c_void_p * len(tensors))(*[_ptr(t) for t in tensors])
        _check(lib.asr_load_weights(self.h, arr, len(tensors), int(on_device)))

    # -- queue ----------------------------------------------------------------
    def set_policy(self, policy, kappa_num=0, kappa_den=0):
        _check(lib.asr_set_policy(self.h, policy, kappa_num, kappa_den))

    def submit(self, rid, pcm, n_samples=None, sample_rate=16000, duration_us=0, arrival_us=0,
               max_tokens=0, on_device=False):
        if pcm is not None and n_samples is None:
            n_samples = pcm.numel() if hasattr(pcm, "numel") else len(pcm)
        if pcm is not None and not on_device:
            pcm = np.ascontiguousarray(pcm, dtype=np.float32)
        _check(lib.asr_submit(self.h, rid, _ptr(pcm) if pcm is not None else None, n_samples,
                              sample_rate, duration_us, arrival_us, max_tokens, int(on_device)))

    def rank(self, now_us, cap=1 << 20):
        n = C.c_int32()
        out = np.zeros(max(cap, 1), np.int64)
        _check(lib.asr_rank(self.h, now_us, out.ctypes.data_as(C.POINTER(C.c_int64)), cap,
                            C.byref(n)))
        return out[:n.value].tolist()

    def pop_batch(self, now_us, max_n):
        n = C.c_int32()
        out = np.zeros(max(max_n, 1), np.int64)
        _check(lib.asr_pop_batch(self.h, now_us, max_n,
                                 out.ctypes.data_as(C.POINTER(C.c_int64)), C.byref(n)))
        return out[:n.value].tolist()

    def queue_len(self):
        n = C.c_int32()
        _check(lib.asr_queue_len(self.h, C.byref(n)))
        return n.value

    # -- step -----------------------------------------------------------------
    def step(self, prefill_ids=(), slots=(), tokens=(), want_logits=False, topk=0):
        """Returns dict(slot_of, argmax, done, logits); with topk also top_token and top_logprob
        [rows][topk] (see asr_step_topk).  Where a row has no next token (its rules allow none, or
        its logits hold a NaN) the slots are a step further all the same: the AsrError's `results`
        are this dict, of every row."""
        pids, p_pids = _i64(list(prefill_ids) or [0])
        sl, p_sl = _i32(list(slots) or [0])
        tk, p_tk = _i32(list(tokens) or [0])
        P, D = len(prefill_ids), len(slots)
        slot_of, p_so = _i32(np.zeros(max(P, 1)))
        am, p_am = _i32(np.full(max(D, 1), NOT_WRITTEN))
        done, p_dn = _i32(np.zeros(max(D, 1)))
        logits = None
        p_lg = None
        if want_logits and D > 0:
            logits = np.zeros((D, self.cfg.vocab), np.float32)
            p_lg = logits.ctypes.data_as(C.POINTER(C.c_float))
        sin = StepIn(P, p_pids, D, p_sl, p_tk, p_lg)
        sout = StepOut(p_so, p_am, p_dn)
        out = {}
        if topk:
            top = np.zeros((max(D, 1), topk), np.int32)
            logp = np.zeros((max(D, 1), topk), np.float32)
            status = lib.asr_step_topk(self.h, C.byref(sin), C.byref(sout), topk,
                                       top.ctypes.data_as(C.POINTER(C.c_int32)),
                                       logp.ctypes.data_as(C.POINTER(C.c_float)))
            out = {"top_token": top[:D], "top_logprob": logp[:D]}
        else:
            status = lib.asr_step(self.h, C.byref(sin), C.byref(sout))
        results = {"slot_of": slot_of[:P].copy(), "argmax": am[:D].copy(),
                   "done": done[:D].astype(bool), "logits": logits, **out}
        _check(status, results if D > 0 and (am[:D] != NOT_WRITTEN).all() else None)
        return results

    # -- hypotheses and rules ---------------------------------------------------
    def hypotheses_size(self, max_bias=0, n_masks=0) -> int:
        n = C.c_size_t()
        _check(lib.asr_hypotheses_size(self.h, max_bias, n_masks, C.byref(n)))
        return n.value

    def bind_hypotheses(self, max_bias=0, n_masks=0, block=None):
        """Binds the block that forked slots and rules need (allocated here when None)."""
        import torch
        if block is None:
            block = torch.empty(self.hypotheses_size(max_bias, n_masks), dtype=torch.uint8,
                                device=f"cuda:{self.device}")
        _check(lib.asr_bind_hypotheses(self.h, max_bias, n_masks, C.c_void_p(block.data_ptr()),
                                       block.numel()))
        self._hyp_block = block
        return block

    def fork_slot(self, src, dst):
        """Makes dst a hypothesis of src's sequence (asr_fork_slot)."""
        _check(lib.asr_fork_slot(self.h, src, dst))

    def set_masks(self, first, allowed):
        """Rows of the mask table from a bool array [n][vocab] of allowed tokens."""
        allowed = np.atleast_2d(np.asarray(allowed, bool))
        n, V = allowed.shape
        if V != self.cfg.vocab:
            raise ValueError(f"masks must cover the vocabulary of {self.cfg.vocab}")
        bits = np.zeros((n, (V + 31) // 32 * 32), np.uint8)
        bits[:, :V] = allowed
        words = np.ascontiguousarray(np.packbits(bits, axis=1, bitorder="little"))
        _check(lib.asr_set_masks(self.h, first, n, words.ctypes.data))

    def set_slot_rules(self, slot, repetition=1.0, frequency=0.0, presence=0.0, temperature=1.0,
                       n_prompt=0, mask=-1, bias=()):
        """Rules of a slot (-1: of every slot filled from now on); bias: (token, value) pairs."""
        bias = list(bias)
        tok, p_tok = _i32([t for t, _ in bias] or [0])
        val = np.ascontiguousarray([v for _, v in bias] or [0.0], dtype=np.float32)
        r = SlotRules(repetition, frequency, presence, temperature, n_prompt, mask, len(bias),
                      p_tok, val.ctypes.data_as(C.POINTER(C.c_float)))
        _check(lib.asr_set_slot_rules(self.h, slot, C.byref(r)))

    def clear_slot_rules(self, slot):
        _check(lib.asr_set_slot_rules(self.h, slot, None))

    def set_slot_mask(self, slot, mask):
        """The row of the mask table that a slot's next tokens must follow (-1: none)."""
        _check(lib.asr_set_slot_mask(self.h, slot, mask))

    def release_slot(self, slot):
        _check(lib.asr_release_slot(self.h, slot))

    # -- continuous batching ----------------------------------------------------
    def serve_config(self, kv_capacity=0, cross_tokens=1500, max_admit=1, tok_num=27,
                     tok_den=10, start_token=0, dynamic=False, depth_low=0, starve=(0, 1),
                     overlap=False):
        """starve = (num, den): the response-ratio threshold of the dynamic rule;
        overlap: prefill on a second stream beside the running rows' decode."""
        cfg = ServeCfg(kv_capacity, cross_tokens, max_admit, tok_num, tok_den, start_token,
                       int(dynamic), depth_low, starve[0], starve[1], int(overlap))  # >1: CUs kept free
        _check(lib.asr_serve_config(self.h, C.byref(cfg)))
        self._serve_cap = max(self.cfg.max_slots, 1)

    def _serve(self, fn, now_us):
        cap = self._serve_cap
        bufs = {k: np.zeros(cap, np.int64) for k in ("preempted", "admitted", "decoded", "finished")}
        slot = np.zeros(cap, np.int32)
        tok = np.zeros(cap, np.int32)
        p64 = lambda a: a.ctypes.data_as(C.POINTER(C.c_int64))  # noqa: E731
        p32 = lambda a: a.ctypes.data_as(C.POINTER(C.c_int32))  # noqa: E731
        out = ServeOut(cap, NOT_WRITTEN, p64(bufs["preempted"]), 0, p64(bufs["admitted"]), p32(slot), 0,
                       p64(bufs["decoded"]), p32(tok), 0, p64(bufs["finished"]), 0)
        status = fn(self.h, now_us, C.byref(out))
        results = {"policy": out.policy,
                   "preempted": bufs["preempted"][:out.n_preempted].tolist(),
                   "admitted": bufs["admitted"][:out.n_admitted].tolist(),
                   "admitted_slot": slot[:out.n_admitted].tolist(),
                   "decoded": bufs["decoded"][:out.n_decoded].tolist(),
                   "token": tok[:out.n_decoded].tolist(),
                   "finished": bufs["finished"][:out.n_finished].tolist()}
        _check(status, results if out.policy != NOT_WRITTEN else None)
        return results

    def serve_step(self, now_us):
        """One continuous-batching step on the GPU (see asr_serve_step).  Where a request ended with
        a NaN logit, the AsrError's `results` are what this returns otherwise."""
        return self._serve(lib.asr_serve_step, now_us)

    def serve_plan(self, now_us):
        """The same schedule without the model (queue-only contexts)."""
        return self._serve(lib.asr_serve_plan, now_us)

    def serve_simulate(self, ids, prefill_us, step_us, row_us, t0_us=0, want_token_times=True,
                       token_cap=None):
        """Virtual-clock serving run (asr_serve_simulate).  Returns
        ({id: {first_us, finish_us, n_tokens, n_preempt, token_us}}, t_end_us)."""
        n = len(ids)
        ids_a = np.asarray(ids, np.int64)
        first = np.zeros(max(n, 1), np.int64)
        fin = np.zeros(max(n, 1), np.int64)
        ntok = np.zeros(max(n, 1), np.int32)
        npre = np.zeros(max(n, 1), np.int32)
        cap = token_cap if token_cap is not None else 448 * max(n, 1)
        tok = np.zeros(cap, np.int64) if want_token_times else None
        t_end = C.c_int64()
        p64 = lambda a: a.ctypes.data_as(C.POINTER(C.c_int64))  # noqa: E731
        p32 = lambda a: a.ctypes.data_as(C.POINTER(C.c_int32))  # noqa: E731
        cost = SimCost(prefill_us, step_us, row_us)
        _check(lib.asr_serve_simulate(self.h, C.byref(cost), t0_us, n, p64(ids_a), p64(first),
                                      p64(fin), p32(ntok), p32(npre),
                                      p64(tok) if tok is not None else None, cap,
                                      C.byref(t_end)))
        out, off = {}, 0
        for i, rid in enumerate(ids):
            k = int(ntok[i])
            out[int(rid)] = {"first_us": int(first[i]), "finish_us": int(fin[i]), "n_tokens": k,
                             "n_preempt": int(npre[i]),
                             "token_us": tok[off:off + k].tolist() if tok is not None else None}
            off += k
        return out, t_end.value

    def serve_stats(self):
        """Steps run under FCFS, SJF and HRRN since serve_config."""
        a = (C.c_int64 * 3)()
        _check(lib.asr_serve_stats(self.h, a))
        return list(a)

    def serve_tokens(self, rid):
        buf = np.zeros(448, np.int32)
        n = C.c_int32()
        _check(lib.asr_serve_tokens(self.h, rid, buf.ctypes.data_as(C.POINTER(C.c_int32)), 448,
                                    C.byref(n)))
        return buf[:n.value].tolist()

    def slot_info(self, slot):
        occ, rid, pos, left = C.c_int32(), C.c_int64(), C.c_int32(), C.c_int32()
        _check(lib.asr_slot_info(self.h, slot, C.byref(occ), C.byref(rid), C.byref(pos),
                                 C.byref(left)))
        return {"occupied": bool(occ.value), "id": rid.value, "position": pos.value,
                "steps_left": left.value}

    def set_encoder_streams(self, n):
        """Prefill clips in n groups whose encoder layers run on n streams."""
        _check(lib.asr_set_encoder_streams(self.h, int(n)))

    # -- timing ---------------------------------------------------------------
    def set_decode_graphs(self, on: bool):
        """Replay decode steps from HIP graphs (default) or launch directly."""
        _check(lib.asr_set_decode_graphs(self.h, int(bool(on))))

    def set_timing(self, classes=True):
        """True times every kernel class, False none; an int is a bit mask
        over the class numbers (K_MEL .. K_DECODE)."""
        if classes is True:
            classes = TIME_ALL
        elif classes is False:
            classes = 0
        _check(lib.asr_set_timing(self.h, int(classes)))

    def reset_timing(self):
        _check(lib.asr_reset_timing(self.h))

    def timing(self):
        out = {}
        for k, name in enumerate(KERNEL_CLASSES):
            ms, n, fl, by = C.c_double(), C.c_int64(), C.c_double(), C.c_double()
            _check(lib.asr_get_timing(self.h, k, C.byref(ms), C.byref(n), C.byref(fl),
                                      C.byref(by)))
            out[name] = {"ms": ms.value, "launches": n.value, "flops": fl.value,
                         "bytes": by.value}
        return out

    # -- debug / parity -------------------------------------------------------
    def _clip_args(self, clips, on_device):
        ptrs = (C.c_void_p * len(clips))(*[_ptr(x) for x in clips])
        ns = np.array([x.numel() if hasattr(x, "numel") else len(x) for x in clips], np.int64)
        return ptrs, ns

    def debug_logmel(self, clips, on_device=False):
        if not on_device:
            clips = [np.ascontiguousarray(x, np.float32) for x in clips]
        ptrs, ns = self._clip_args(clips, on_device)
        out = np.zeros((len(clips), 3000, self.cfg.n_mels), np.float32)
        _check(lib.asr_debug_logmel(self.h, ptrs, ns.ctypes.data_as(C.POINTER(C.c_int64)),
                                    len(clips), int(on_device),
                                    out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def debug_encode(self, clips, on_device=False):
        if not on_device:
            clips = [np.ascontiguousarray(x, np.float32) for x in clips]
        ptrs, ns = self._clip_args(clips, on_device)
        out = np.zeros((len(clips), 1500, self.cfg.d_model), np.float32)
        _check(lib.asr_debug_encode(self.h, ptrs, ns.ctypes.data_as(C.POINTER(C.c_int64)),
                                    len(clips), int(on_device),
                                    out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def debug_attention(self, q, k, v):
        """Encoder attention kernel on [n][1500][d] operands; q in the exp2
        domain (queries times 1/sqrt(64) log2(e))."""
        q, k, v = (np.ascontiguousarray(x, np.float32) for x in (q, k, v))
        assert q.shape == k.shape == v.shape and q.shape[1:] == (1500, self.cfg.d_model)
        out = np.zeros(q.shape, np.float32)
        fp = C.POINTER(C.c_float)
        _check(lib.asr_debug_attention(self.h, q.ctypes.data_as(fp), k.ctypes.data_as(fp),
                                       v.ctypes.data_as(fp), q.shape[0], out.ctypes.data_as(fp)))
        return out

    def debug_set_encoder_out(self, slots, ids, steps_left, E, on_device=False):
        sl, p_sl = _i32(slots)
        idv, p_id = _i64(ids)
        st, p_st = _i32(steps_left)
        if not on_device:
            E = np.ascontiguousarray(E, np.float32)
        _check(lib.asr_debug_set_encoder_out(self.h, p_sl, p_id, p_st, len(sl), _ptr(E),
                                             int(on_device)))

    def debug_get_kv(self, slot, which):
        H = self.cfg.n_head
        ctx = 448 if which == 0 else 1500
        out = np.zeros((self.cfg.n_dec, 2, H, ctx, 64), np.float32)
        _check(lib.asr_debug_get_kv(self.h, slot, which, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def debug_set_self_kv(self, slot, src, length, on_device=False):
        if not on_device:
            src = np.ascontiguousarray(src, np.float32)
        _check(lib.asr_debug_set_self_kv(self.h, slot, _ptr(src), length, int(on_device)))
