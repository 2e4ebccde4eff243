"""Python binding of libparason.so (argument marshalling only).

Every step of the path runs in the HIP kernels behind the C-ABI declared in
``include/parason.h``; this module turns torch tensors into device pointers and
passes torch's current HIP stream.  It raises if the library is missing: there
is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Any, NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libparason.so")

OK = 0
ERR_NULL, ERR_SIZE, ERR_GROUP, ERR_WORKSPACE, ERR_TAGS, ERR_PARAM, ERR_ALIGN, ERR_HIP, ERR_DEVICE, ERR_SCRATCH = \
    range(-1, -11, -1)
NOALLOC_SCRATCH_BYTES = 128 << 20

FLAG_VALID = 1 << 0
FLAG_TRUNCATED = 1 << 1
FLAG_COUNT_MISMATCH = 1 << 2
FLAG_TRIGGERED = 1 << 3
FLAG_DEPTH_LIMIT = 1 << 8
FLAG_WS_OVERFLOW = 1 << 9
FLAG_BAD_ROW = 1 << 10

CFG_INVALID_KEEPS_CORRECTNESS = 1 << 0
CFG_BATCH_STATS = 1 << 1
CFG_TAG_COMPARE = 1 << 2
CFG_LENIENT_GAPS = 1 << 3

METRICS = (
    "rows", "valid", "triggered", "correct", "truncated", "count_mismatch",
    "sum_total", "sum_latency", "sum_subtask", "sum_trial",
    "trigger_ratio", "acceleration", "mean_latency", "mean_total", "mean_saved",
    "subtask_share", "trial_share", "accuracy", "mean_reward",
)

MAX_DEPTH = 1 << 20
MAX_OPEN_ENTRIES = 1 << 24

EXPORTED = ("parason_create", "parason_workspace_size", "parason_run", "parason_run_timed", "parason_destroy",
            "parason_strerror", "parason_pg_workspace_size", "parason_pg_run", "parason_decode_init",
            "parason_decode_step", "parason_fork_workspace_size", "parason_join_workspace_size", "parason_fork",
            "parason_join", "parason_read_probe", "parason_run_noalloc", "parason_fork_sized", "parason_join_sized",
            "parason_kv_write", "parason_kv_read", "parason_tree_attention_workspace_size", "parason_tree_attention",
            "parason_beam_workspace_size", "parason_beam_select", "parason_beam_reorder")

FORK_SEED_ENTRY = 1 << 0
JOIN_CLOSE_PARALLEL = 1 << 0
JOIN_APPEND_ONLY = 1 << 1
PACK_NO_OUTLINE_END = 1 << 0
PACK_NO_OUTLINE = 1 << 1
PACK_BAD_ENTRY = 1 << 2
PACK_BAD_THREAD = 1 << 3
PACK_TOO_LONG = 1 << 4
PACK_BAD_ROW = 1 << 5

DECODE_ERROR = 1 << 0
DECODE_DONE = 1 << 1
DTYPE_F32, DTYPE_BF16, DTYPE_F16, DTYPE_FP8, DTYPE_INT8 = range(5)
DECODE_STATE_BYTES = 16

KV_BAD_ROW = 1 << 0
KV_BAD_PAGE = 1 << 1
KV_MAX_DIM = 256
KV_MAX_HEADS = 1024
KV_MAX_LEN = 1 << 30
BEAM_MAX = 64
BEAM_ARRAYS = 8

PG_STATS = ("loss", "tokens", "clip_high", "clip_low")


class Config(ctypes.Structure):
    _fields_ = [
        ("tag_ids", ctypes.c_int32 * 12),
        ("group_size", ctypes.c_int32),
        ("alpha", ctypes.c_double),
        ("beta_subtask", ctypes.c_double),
        ("beta_trial", ctypes.c_double),
        ("rho", ctypes.c_double),
        ("rho_clip", ctypes.c_double),
        ("flags", ctypes.c_uint32),
    ]


class PgConfig(ctypes.Structure):
    _fields_ = [("group_size", ctypes.c_int32), ("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double)]


class Outputs(ctypes.Structure):
    _fields_ = [
        ("total", ctypes.c_void_p),
        ("latency", ctypes.c_void_p),
        ("n_subtask", ctypes.c_void_p),
        ("n_trial", ctypes.c_void_p),
        ("n_blocks", ctypes.c_void_p),
        ("max_depth", ctypes.c_void_p),
        ("first_error_pos", ctypes.c_void_p),
        ("flags", ctypes.c_void_p),
        ("reward", ctypes.c_void_p),
        ("r_subtask", ctypes.c_void_p),
        ("r_trial", ctypes.c_void_p),
        ("eta", ctypes.c_void_p),
        ("metrics", ctypes.c_void_p),
        ("accel", ctypes.c_void_p),
        ("saved", ctypes.c_void_p),
    ]


class ForkOutputs(ctypes.Structure):
    _fields_ = [
        ("max_workers", ctypes.c_int64),
        ("ctx_capacity", ctypes.c_int64),
        ("ctx_tokens", ctypes.c_void_p),
        ("ctx_starts", ctypes.c_void_p),
        ("ctx_lengths", ctypes.c_void_p),
        ("ctx_row", ctypes.c_void_p),
        ("ctx_entry", ctypes.c_void_p),
        ("ctx_kind", ctypes.c_void_p),
        ("worker_off", ctypes.c_void_p),
        ("row_status", ctypes.c_void_p),
        ("totals", ctypes.c_void_p),
    ]


class JoinOutputs(ctypes.Structure):
    _fields_ = [
        ("capacity", ctypes.c_int64),
        ("tokens", ctypes.c_void_p),
        ("starts", ctypes.c_void_p),
        ("lengths", ctypes.c_void_p),
        ("row_status", ctypes.c_void_p),
        ("totals", ctypes.c_void_p),
    ]


class KvCacheArgs(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("n_pages", ctypes.c_int64),
        ("stride_page", ctypes.c_int64),
        ("stride_slot", ctypes.c_int64),
        ("stride_head", ctypes.c_int64),
        ("scale_stride_page", ctypes.c_int64),
        ("scale_stride_slot", ctypes.c_int64),
        ("scale_stride_head", ctypes.c_int64),
        ("page_size", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
    ]


class KvRowsArgs(ctypes.Structure):
    _fields_ = [
        ("n_rows", ctypes.c_int64),
        ("n_tokens", ctypes.c_int64),
        ("starts", ctypes.c_void_p),
        ("lengths", ctypes.c_void_p),
        ("kv_lens", ctypes.c_void_p),
        ("pages", ctypes.c_void_p),
        ("pages_stride", ctypes.c_int64),
        ("max_pages", ctypes.c_int32),
        ("max_length", ctypes.c_int32),
        ("max_kv_len", ctypes.c_int32),
    ]


class TreeArgs(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p),
        ("out", ctypes.c_void_p),
        ("lse", ctypes.c_void_p),
        ("q_stride_token", ctypes.c_int64),
        ("q_stride_head", ctypes.c_int64),
        ("out_stride_token", ctypes.c_int64),
        ("out_stride_head", ctypes.c_int64),
        ("mask", ctypes.c_void_p),
        ("mask_stride", ctypes.c_int64),
        ("tree_lens", ctypes.c_void_p),
        ("mask_words", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]


class BeamArray(ctypes.Structure):
    _fields_ = [
        ("src", ctypes.c_void_p),
        ("dst", ctypes.c_void_p),
        ("row_bytes", ctypes.c_int64),
        ("src_stride", ctypes.c_int64),
        ("dst_stride", ctypes.c_int64),
    ]


INT_FIELDS = ("total", "latency", "n_subtask", "n_trial", "n_blocks", "max_depth", "first_error_pos")
FLOAT_FIELDS = ("reward", "r_subtask", "r_trial", "eta", "accel")
OPTIONAL_FIELDS = ("r_subtask", "r_trial", "eta", "metrics", "accel", "saved")  # in the order of Outputs

_OUT_FIELDS = INT_FIELDS + ("flags", "reward")  # required, in the order of Outputs

_lib = None


def _stream(device) -> int:
    """The raw handle of torch's current stream on `device`.  (A Stream object
    for every call would cost more than the rest of its arguments.)"""
    import torch

    return torch._C._cuda_getCurrentRawStream(device.index)


def _outputs(out: dict) -> Outputs:
    get = out.get
    ptrs = [out[k].data_ptr() for k in _OUT_FIELDS]
    for k in OPTIONAL_FIELDS:
        t = get(k)
        ptrs.append(t.data_ptr() if t is not None else None)
    return Outputs(*ptrs)


class ParasonError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (what, strerror(status), status))


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libparason.so is not built (%s); run __graft_entry__.build() -- there is no fallback" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        L.parason_create.restype = ctypes.c_int
        L.parason_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(ctypes.c_void_p)]
        L.parason_workspace_size.restype = ctypes.c_int
        L.parason_workspace_size.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]
        L.parason_run.restype = ctypes.c_int
        L.parason_run.argtypes = [
            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
            ctypes.POINTER(Outputs), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
        ]
        L.parason_run_noalloc.restype = ctypes.c_int
        L.parason_run_noalloc.argtypes = [
            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
            ctypes.c_int64, ctypes.POINTER(Outputs), ctypes.c_void_p,
        ]
        L.parason_run_timed.restype = ctypes.c_int
        L.parason_run_timed.argtypes = L.parason_run.argtypes + [ctypes.c_void_p]
        L.parason_destroy.restype = None
        L.parason_destroy.argtypes = [ctypes.c_void_p]
        L.parason_pg_workspace_size.restype = ctypes.c_int
        L.parason_pg_workspace_size.argtypes = [ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]
        L.parason_pg_run.restype = ctypes.c_int
        L.parason_pg_run.argtypes = [
            ctypes.POINTER(PgConfig), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
            ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
            ctypes.c_size_t, ctypes.c_void_p,
        ]
        L.parason_decode_init.restype = ctypes.c_int
        L.parason_decode_init.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]
        L.parason_decode_step.restype = ctypes.c_int
        L.parason_decode_step.argtypes = [
            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
            ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
        ]
        for name in ("parason_fork_workspace_size", "parason_join_workspace_size"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = [ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]
        for name in ("parason_fork", "parason_fork_sized"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = [
                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint32,
                ctypes.POINTER(ForkOutputs), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
            ]
        for name in ("parason_join", "parason_join_sized"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = [
                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint32,
                ctypes.POINTER(JoinOutputs), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
            ]
        L.parason_read_probe.restype = ctypes.c_int
        L.parason_read_probe.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int64,
                                         ctypes.c_void_p]
        cache, rows, void, i64 = ctypes.POINTER(KvCacheArgs), ctypes.POINTER(KvRowsArgs), ctypes.c_void_p, ctypes.c_int64
        for name, args in (
            ("parason_kv_write", [cache, rows, void, void, ctypes.c_int32, i64, i64, void, void]),
            ("parason_kv_read", [cache, rows, void, void, ctypes.c_int32, i64, i64, void, void]),
            ("parason_tree_attention_workspace_size", [cache, rows, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]),
            ("parason_tree_attention", [cache, rows, ctypes.POINTER(TreeArgs), void, void, ctypes.c_size_t, void]),
            ("parason_beam_workspace_size", [i64, ctypes.c_int32, i64, ctypes.POINTER(ctypes.c_size_t)]),
            ("parason_beam_select", [void, i64, i64, ctypes.c_int32, void, void, i64, ctypes.c_int32, void, void, void,
                                     void, ctypes.c_size_t, void]),
            ("parason_beam_reorder", [void, i64, ctypes.POINTER(BeamArray), ctypes.c_int32, void]),
        ):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = args
        L.parason_strerror.restype = ctypes.c_char_p
        L.parason_strerror.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().parason_strerror(status).decode()


def make_config(tag_ids, group_size=8, alpha=0.1, beta_subtask=0.0, beta_trial=0.1, rho=0.5, rho_clip=0.25,
                flags=0) -> Config:
    c = Config()
    ids = [int(t) for t in tag_ids]
    if len(ids) != 12:
        raise ValueError("tag_ids must have 12 entries")
    for i, t in enumerate(ids):
        c.tag_ids[i] = t
    c.group_size = int(group_size)
    c.alpha, c.beta_subtask, c.beta_trial = float(alpha), float(beta_subtask), float(beta_trial)
    c.rho, c.rho_clip = float(rho), float(rho_clip)
    c.flags = int(flags)
    return c


class Parason:
    """Handle of the C-ABI (immutable configuration)."""

    def __init__(self, tag_ids, group_size=8, alpha=0.1, beta_subtask=0.0, beta_trial=0.1, rho=0.5,
                 rho_clip=0.25, flags=0):
        self.config = make_config(tag_ids, group_size, alpha, beta_subtask, beta_trial, rho, rho_clip, flags)
        h = ctypes.c_void_p()
        rc = lib().parason_create(ctypes.byref(self.config), ctypes.byref(h))
        if rc != OK:
            raise ParasonError(rc, "parason_create")
        self._h = h

    @property
    def group_size(self) -> int:
        return self.config.group_size

    def close(self):
        if getattr(self, "_h", None):
            lib().parason_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_size(self, n_traj: int, total_tokens: int) -> int:
        b = ctypes.c_size_t()
        rc = lib().parason_workspace_size(self._h, int(n_traj), int(total_tokens), ctypes.byref(b))
        if rc != OK:
            raise ParasonError(rc, "parason_workspace_size")
        return b.value

    def alloc_outputs(self, n_traj: int, device, derived: bool = True, metrics: bool = False) -> dict:
        import torch

        out = {k: torch.empty(n_traj, dtype=torch.int32, device=device) for k in INT_FIELDS}
        out["flags"] = torch.empty(n_traj, dtype=torch.int32, device=device)  # uint32 bits
        out["reward"] = torch.empty(n_traj, dtype=torch.float32, device=device)
        if derived:
            for k in ("r_subtask", "r_trial", "eta", "accel"):
                out[k] = torch.empty(n_traj, dtype=torch.float32, device=device)
            out["saved"] = torch.empty(n_traj, dtype=torch.int32, device=device)
        if metrics:
            out["metrics"] = torch.empty(len(METRICS), dtype=torch.float64, device=device)
        return out

    def alloc_workspace(self, n_traj: int, total_tokens: int, device):
        import torch

        return torch.empty(self.workspace_size(n_traj, total_tokens), dtype=torch.uint8, device=device)

    def run_raw(self, tokens_ptr, starts_ptr, lengths_ptr, correct_ptr, n_traj, out: dict, ws_ptr, ws_bytes,
                stream) -> int:
        """Direct C-ABI call with raw device pointers; returns the status."""
        o = _outputs(out)
        return lib().parason_run(self._h, tokens_ptr, starts_ptr, lengths_ptr, correct_ptr, int(n_traj),
                                 ctypes.byref(o), ws_ptr, int(ws_bytes), stream)

    def run_noalloc_raw(self, tokens_ptr, starts_ptr, lengths_ptr, correct_ptr, n_traj, total_tokens, out: dict,
                        stream) -> int:
        """parason_run_noalloc (no workspace: the library's static scratch); returns the status."""
        o = _outputs(out)
        return lib().parason_run_noalloc(self._h, tokens_ptr, starts_ptr, lengths_ptr, correct_ptr, int(n_traj),
                                         int(total_tokens), ctypes.byref(o), stream)

    def run_timed_raw(self, tokens_ptr, starts_ptr, lengths_ptr, correct_ptr, n_traj, out: dict, ws_ptr, ws_bytes,
                      stream, scan_events) -> int:
        """parason_run_timed: scan_events is a ctypes array of two hipEvent_t (or None)."""
        o = _outputs(out)
        ev = ctypes.cast(scan_events, ctypes.c_void_p) if scan_events is not None else None
        return lib().parason_run_timed(self._h, tokens_ptr, starts_ptr, lengths_ptr, correct_ptr, int(n_traj),
                                       ctypes.byref(o), ws_ptr, int(ws_bytes), stream, ev)

    def decode_step_raw(self, states_ptr, tokens_ptr, batch, logits_ptr, vocab, row_stride, dtype, eos_id,
                        stream) -> int:
        """Direct parason_decode_step call with raw device pointers; returns the status."""
        return lib().parason_decode_step(self._h, states_ptr, tokens_ptr, int(batch), logits_ptr, int(vocab),
                                         int(row_stride), int(dtype), int(eos_id), stream)

    def decode_step(self, states, logits, tokens=None, eos_id: int = -1):
        """Advance the decode states by `tokens` (int32[batch] or None) and mask
        `logits` ([batch, vocab] rows, float32/bfloat16/float16, unit stride
        along the vocabulary) in place, on the current stream."""
        import torch

        dtype = logits.dtype
        code = (DTYPE_BF16 if dtype is torch.bfloat16 else DTYPE_F32 if dtype is torch.float32
                else DTYPE_F16 if dtype is torch.float16 else None)
        if code is None or logits.dim() != 2 or logits.stride(1) != 1 or not logits.is_cuda:
            raise TypeError("logits must be a [batch, vocab] float32/bfloat16/float16 device tensor, unit stride")
        batch, vocab = logits.shape
        if states.dtype != torch.uint8 or states.numel() != batch * DECODE_STATE_BYTES or not states.is_contiguous():
            raise TypeError("states must be a contiguous uint8 device tensor of batch * 16 bytes")
        if tokens is not None and (tokens.dtype != torch.int32 or tokens.numel() != batch
                                   or not tokens.is_contiguous()):
            raise TypeError("tokens must be a contiguous int32 device tensor of batch entries")
        rc = (_lib or lib()).parason_decode_step(
            self._h, states.data_ptr(), tokens.data_ptr() if tokens is not None else None, batch, logits.data_ptr(),
            vocab, logits.stride(0) if batch > 1 else vocab, code, int(eos_id), _stream(logits.device))
        if rc != OK:
            raise ParasonError(rc, "parason_decode_step")
        return logits

    def fork_raw(self, tokens_ptr, starts_ptr, lengths_ptr, n_rows, flags, out: ForkOutputs, ws_ptr, ws_bytes,
                 stream, sized: bool = False) -> int:
        """parason_fork, or parason_fork_sized right after a sizing call."""
        fn = lib().parason_fork_sized if sized else lib().parason_fork
        return fn(self._h, tokens_ptr, starts_ptr, lengths_ptr, int(n_rows), int(flags), ctypes.byref(out), ws_ptr,
                  int(ws_bytes), stream)

    def join_raw(self, tokens_ptr, starts_ptr, lengths_ptr, n_rows, worker_off_ptr, wtokens_ptr, wstarts_ptr,
                 wlengths_ptr, n_workers, flags, out: JoinOutputs, ws_ptr, ws_bytes, stream,
                 sized: bool = False) -> int:
        """parason_join, or parason_join_sized right after a sizing call."""
        fn = lib().parason_join_sized if sized else lib().parason_join
        return fn(self._h, tokens_ptr, starts_ptr, lengths_ptr, int(n_rows), worker_off_ptr, wtokens_ptr, wstarts_ptr,
                  wlengths_ptr, int(n_workers), int(flags), ctypes.byref(out), ws_ptr, int(ws_bytes), stream)

    def fork(self, tokens, starts, lengths, seed: bool = True, max_workers=None, ctx_capacity=None) -> dict:
        """Worker contexts of a batch of rows (device tensors).  Without
        capacities, a first call sizes the outputs (one synchronisation)."""
        import torch

        _check_rows(tokens, starts, lengths)
        dev, n = starts.device, starts.numel()
        flags = FORK_SEED_ENTRY if seed else 0
        ws = torch.empty(_ws_size("parason_fork_workspace_size", n), dtype=torch.uint8, device=dev)
        stream = _stream(dev)
        i64, i32 = starts.new_empty, lengths.new_empty  # int64, int32 on the rows' device
        worker_off, row_status, totals = i64(n + 1), i32(n), i64(3)
        rows = (_ptr(tokens, starts), starts.data_ptr(), lengths.data_ptr(), n, flags)
        res = dict(worker_off=worker_off, row_status=row_status, totals=totals)
        tail = (worker_off.data_ptr(), row_status.data_ptr() if n else None, totals.data_ptr())

        def call(W, T, sized=False):
            if W or T:
                res.update(ctx_tokens=i32(T), ctx_starts=i64(W), ctx_lengths=i32(W), ctx_row=i32(W), ctx_entry=i32(W),
                           ctx_kind=i32(W))
            elif sized or not sizing:
                res.update(ctx_tokens=i32(0), ctx_starts=i64(0), ctx_lengths=i32(0), ctx_row=i32(0), ctx_entry=i32(0),
                           ctx_kind=i32(0))
            ctx = [res[k].data_ptr() or None for k in (
                "ctx_tokens", "ctx_starts", "ctx_lengths", "ctx_row", "ctx_entry", "ctx_kind")] if W or T else [None] * 6
            rc = self.fork_raw(*rows, ForkOutputs(W, T, *ctx, *tail), ws.data_ptr(), ws.numel(), stream, sized)
            if rc != OK:
                raise ParasonError(rc, "parason_fork")

        sizing = max_workers is None or ctx_capacity is None
        if sizing:
            call(0, 0)
            W, T, _ = res["totals"].tolist()
            max_workers = W if max_workers is None else max_workers
            ctx_capacity = T if ctx_capacity is None else ctx_capacity
        call(int(max_workers), int(ctx_capacity), sizing)
        return res

    def join(self, tokens, starts, lengths, worker_off, wtokens, wstarts, wlengths, close: bool = True,
             append_only: bool = False, capacity=None) -> dict:
        """Joined rows (device tensors); sizing as for fork."""
        import torch

        _check_rows(tokens, starts, lengths)
        _check_rows(wtokens, wstarts, wlengths)
        dev, n, nw = starts.device, starts.numel(), wstarts.numel()
        flags = (JOIN_CLOSE_PARALLEL if close else 0) | (JOIN_APPEND_ONLY if append_only else 0)
        ws = torch.empty(_ws_size("parason_join_workspace_size", n), dtype=torch.uint8, device=dev)
        stream = _stream(dev)
        i64, i32 = starts.new_empty, lengths.new_empty  # int64, int32 on the rows' device
        res = dict(starts=i64(n + 1), lengths=i32(n), row_status=i32(n), totals=i64(2))
        args = (_ptr(tokens, starts), starts.data_ptr(), lengths.data_ptr(), n, worker_off.data_ptr(),
                _ptr(wtokens, wstarts), wstarts.data_ptr(), wlengths.data_ptr(), nw, flags)
        tail = [res[k].data_ptr() or None for k in ("starts", "lengths", "row_status", "totals")]

        def call(T, sized=False):
            if T or sized or not sizing:
                res["tokens"] = i32(T)
            o = JoinOutputs(T, res["tokens"].data_ptr() if T else None, *tail)
            rc = self.join_raw(*args, o, ws.data_ptr(), ws.numel(), stream, sized)
            if rc != OK:
                raise ParasonError(rc, "parason_join")

        sizing = capacity is None
        if sizing:
            call(0)
            capacity = res["totals"].tolist()[0]
        call(int(capacity), sizing)
        return res

    def run(self, tokens, starts, lengths, correct, out: dict | None = None, workspace=None, total_tokens=None,
            derived: bool = True, metrics: bool = False) -> dict:
        """Evaluate a batch of rows held in device tensors (asynchronous on the
        current stream).  tokens int32, starts int64, lengths int32, correct uint8."""
        import torch

        n = int(starts.numel())
        for t, dt in ((tokens, torch.int32), (starts, torch.int64), (lengths, torch.int32), (correct, torch.uint8)):
            if t.dtype != dt or not t.is_cuda or not t.is_contiguous():
                raise TypeError("expected contiguous %s device tensors" % dt)
        if lengths.numel() != n or correct.numel() != n:
            raise ValueError("starts, lengths and correct must have the same length")
        if out is None:
            out = self.alloc_outputs(n, tokens.device, derived, metrics)
        if workspace is None:
            if total_tokens is None:
                total_tokens = int(lengths.to(torch.int64).clamp_min(0).sum().item()) if n else 0
            workspace = self.alloc_workspace(n, total_tokens, tokens.device)
        stream = _stream(tokens.device)
        tok_ptr = tokens.data_ptr() if tokens.numel() else starts.data_ptr()
        rc = self.run_raw(tok_ptr, starts.data_ptr(), lengths.data_ptr(), correct.data_ptr(), n, out,
                          workspace.data_ptr(), workspace.numel(), stream)
        if rc != OK:
            raise ParasonError(rc, "parason_run")
        return out


def read_probe_raw(data_ptr, nbytes, sink_ptr, sink_len, stream) -> int:
    """parason_read_probe: streaming read of nbytes at data_ptr (measurement)."""
    return lib().parason_read_probe(data_ptr, int(nbytes), sink_ptr, int(sink_len), stream)


def _check_rows(tokens, starts, lengths):
    import torch

    for t, dt in ((tokens, torch.int32), (starts, torch.int64), (lengths, torch.int32)):
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous():
            raise TypeError("expected contiguous %s device tensors" % dt)
    if starts.numel() != lengths.numel():
        raise ValueError("starts and lengths must have the same length")


def _ptr(tokens, fallback):
    return tokens.data_ptr() if tokens.numel() else fallback.data_ptr()


@functools.lru_cache(maxsize=256)
def _ws_size(name: str, n: int) -> int:
    b = ctypes.c_size_t()
    rc = getattr(lib(), name)(int(n), ctypes.byref(b))
    if rc != OK:
        raise ParasonError(rc, name)
    return b.value


def decode_init(batch: int, device, states=None):
    """Decode states (uint8[batch * 16] device tensor) set to the start of a stream."""
    import torch

    if states is None:
        states = torch.empty(int(batch) * DECODE_STATE_BYTES, dtype=torch.uint8, device=device)
    stream = _stream(states.device)
    rc = lib().parason_decode_init(states.data_ptr(), int(batch), stream)
    if rc != OK:
        raise ParasonError(rc, "parason_decode_init")
    return states


def decode_fields(states):
    """[batch, 4] int32 view of a states tensor: state, depth, entry, flags."""
    import torch

    return states.view(torch.int32).view(-1, 4)


def pg_workspace_size(n_traj: int) -> int:
    return _ws_size("parason_pg_workspace_size", int(n_traj))


def pg_run_raw(cfg: PgConfig, reward_ptr, logp_ptr, old_ptr, starts_ptr, lengths_ptr, n_traj, adv_ptr, grad_ptr,
               stats_ptr, ws_ptr, ws_bytes, stream) -> int:
    return lib().parason_pg_run(ctypes.byref(cfg), reward_ptr, logp_ptr, old_ptr, starts_ptr, lengths_ptr,
                                int(n_traj), adv_ptr, grad_ptr, stats_ptr, ws_ptr, int(ws_bytes), stream)


def pg_run(reward, logp, logp_old, starts, lengths, group_size=8, clip_low=0.2, clip_high=0.28, grad=None,
           workspace=None) -> dict:
    """Advantages, gradient d loss / d logp and the step statistics (device
    tensors; asynchronous on the current stream).  reward float32[n], logp and
    logp_old float32 in the row layout of starts/lengths."""
    import torch

    n = int(starts.numel())
    for t, dt in ((reward, torch.float32), (logp, torch.float32), (logp_old, torch.float32),
                  (starts, torch.int64), (lengths, torch.int32)):
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous():
            raise TypeError("expected contiguous %s device tensors" % dt)
    dev = logp.device
    cfg = PgConfig(int(group_size), float(clip_low), float(clip_high))
    adv = reward.new_empty(n)
    if grad is None:
        grad = torch.empty_like(logp)
    stats = torch.empty(len(PG_STATS), dtype=torch.float64, device=dev)
    if workspace is None:
        workspace = torch.empty(pg_workspace_size(n), dtype=torch.uint8, device=dev)
    stream = _stream(dev)
    rc = pg_run_raw(cfg, reward.data_ptr(), logp.data_ptr(), logp_old.data_ptr(), starts.data_ptr(),
                    lengths.data_ptr(), n, adv.data_ptr(), grad.data_ptr(), stats.data_ptr(), workspace.data_ptr(),
                    workspace.numel(), stream)
    if rc != OK:
        raise ParasonError(rc, "parason_pg_run")
    return dict(advantage=adv, grad=grad, stats=stats)


# ---- the cache of rollouts in progress, tree attention, beams ----------------


class KVCache(NamedTuple):
    """Paged keys and values (device tensors).  k and v are [pages, page_size,
    heads, head_dim] in any layout whose last stride is 1, of one type (bfloat16,
    float16, float8_e4m3fn or int8) and with the same strides; k_scale and
    v_scale (8-bit types only) float32 [pages, page_size, heads], with the same
    strides."""

    k: Any
    v: Any
    k_scale: Any = None
    v_scale: Any = None


class KVRows(NamedTuple):
    """The rows of a call (device tensors): row i has lengths[i] tokens at
    starts[i] of the call's token arrays and kv_lens[i] positions in the cache,
    on the pages pages[i].  starts int64, lengths and kv_lens int32, pages int32
    [rows, max_pages] with unit stride along a row.  max_length and max_kv_len
    are bounds of lengths and kv_lens that the program knows."""

    starts: Any
    lengths: Any
    kv_lens: Any
    pages: Any
    max_length: int
    max_kv_len: int


def kv_alloc(n_pages: int, page_size: int, heads: int, head_dim: int, dtype, device) -> KVCache:
    """A cache of zeros, each head's slots of a page next to each other."""
    import torch

    code = _types().kv.get(dtype)
    if code is None:
        raise TypeError("a cache holds bfloat16, float16, float8_e4m3fn or int8 values")
    shape = (int(n_pages), int(heads), int(page_size), int(head_dim))
    kv = [torch.zeros(shape, dtype=torch.uint8 if code >= DTYPE_FP8 else dtype, device=device).view(dtype)
          .permute(0, 2, 1, 3) for _ in "kv"]
    if code >= DTYPE_FP8:
        kv += [torch.zeros(shape[:3], dtype=torch.float32, device=device).permute(0, 2, 1) for _ in "kv"]
    return KVCache(*kv)


class _Types:
    """torch and its types, looked up once (an import statement in every call costs more than its checks)."""

    torch = None

    @classmethod
    def load(cls):
        import torch

        cls.i32, cls.i64, cls.f32, cls.u8 = torch.int32, torch.int64, torch.float32, torch.uint8
        cls.floats = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}
        cls.kv = {torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16, torch.float8_e4m3fn: DTYPE_FP8, torch.int8: DTYPE_INT8}
        cls.empty, cls.grad_enabled, cls.torch = torch.empty, torch.is_grad_enabled, torch
        return cls


def _types():
    return _Types if _Types.torch is not None else _Types.load()


def _refuse_gradients(T):
    """For inputs that require one: these operators have no backward pass, so a result would silently have none."""
    if T.grad_enabled():
        raise RuntimeError("no gradient flows through the cache and the attention over it: detach the inputs, or call under "
                           "torch.no_grad()")


def _cache_args(T, cache: KVCache) -> KvCacheArgs:
    k, v, ks, vs = cache
    code = T.kv.get(k.dtype)
    if code is None or v.dtype is not k.dtype or k.dim() != 4 or not (k.is_cuda and v.is_cuda):
        raise TypeError("k and v must be [pages, page_size, heads, head_dim] bfloat16/float16/float8_e4m3fn/int8 "
                        "device tensors of one type")
    if k.requires_grad or v.requires_grad:
        _refuse_gradients(T)
    shape, st = k.shape, k.stride()
    pages, size, heads, dim = shape
    if v.shape != shape or v.stride() != st or (st[3] != 1 and dim > 1):
        raise ValueError("k and v must have the same shape and strides, and unit stride along a head")
    if code < DTYPE_FP8:
        if ks is not None or vs is not None:
            raise TypeError("a 16-bit cache has no scales")
        return KvCacheArgs(k.data_ptr(), v.data_ptr(), None, None, pages, st[0], st[1], st[2], 0, 0, 0, size, heads, dim,
                           code)
    if ks is None or vs is None or ks.dtype is not T.f32 or vs.dtype is not T.f32 or not (ks.is_cuda and vs.is_cuda):
        raise TypeError("an 8-bit cache needs float32 device tensors k_scale and v_scale")
    sst = ks.stride()
    if ks.shape != shape[:3] or vs.shape != ks.shape or vs.stride() != sst:
        raise ValueError("k_scale and v_scale must be [pages, page_size, heads], with the same strides")
    return KvCacheArgs(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, st[0], st[1], st[2], *sst, size,
                       heads, dim, code)


def _rows_args(T, rows: KVRows, n_tokens: int) -> KvRowsArgs:
    starts, lengths, kv_lens, pages, max_length, max_kv_len = rows
    if starts.dtype is not T.i64 or lengths.dtype is not T.i32 or kv_lens.dtype is not T.i32 \
            or not (starts.is_cuda and lengths.is_cuda and kv_lens.is_cuda) \
            or not (starts.is_contiguous() and lengths.is_contiguous() and kv_lens.is_contiguous()):
        raise TypeError("starts (int64), lengths and kv_lens (int32) must be contiguous device tensors")
    if pages.dtype is not T.i32 or not pages.is_cuda or pages.dim() != 2:
        raise TypeError("pages must be an int32 [rows, max_pages] device tensor, unit stride along a row")
    n, max_pages = pages.shape
    st = pages.stride()
    if st[1] != 1 and max_pages > 1:
        raise TypeError("pages must be an int32 [rows, max_pages] device tensor, unit stride along a row")
    if starts.numel() != n or lengths.numel() != n or kv_lens.numel() != n:
        raise ValueError("starts, lengths, kv_lens and pages must have the same number of rows")
    return KvRowsArgs(n, n_tokens, starts.data_ptr(), lengths.data_ptr(), kv_lens.data_ptr(), pages.data_ptr(), st[0],
                      max_pages, int(max_length), int(max_kv_len))


def _check_workspace(T, workspace):
    if workspace.dtype is not T.u8 or not workspace.is_contiguous() or not workspace.is_cuda:
        raise TypeError("workspace must be a contiguous uint8 device tensor")


def _status_ptr(T, status, n):
    if status is None:
        return None
    if status.dtype is not T.i32 or status.numel() != n or not status.is_contiguous() or not status.is_cuda:
        raise TypeError("status must be a contiguous int32 device tensor of one entry per row")
    return status.data_ptr()


def _token_arrays(T, k, v, ca: KvCacheArgs):
    """Type, token stride and head stride of two [tokens, heads, head_dim] tensors."""
    code = T.floats.get(k.dtype)
    if code is None or v.dtype is not k.dtype or k.dim() != 3 or not (k.is_cuda and v.is_cuda):
        raise TypeError("k and v must be [tokens, heads, head_dim] float32/bfloat16/float16 device tensors of one type")
    shape, st = k.shape, k.stride()
    if v.shape != shape or v.stride() != st or shape[1] != ca.n_heads or shape[2] != ca.head_dim \
            or (st[2] != 1 and shape[2] > 1):
        raise ValueError("k and v must have the cache's heads, the same shape and strides, and unit stride along a head")
    return code, st[0], st[1]


def kv_write(k, v, cache: KVCache, rows: KVRows, status=None) -> None:
    """Write the keys and values of the rows' tokens ([tokens, heads, head_dim]
    tensors) into the cache, at the last lengths[i] of row i's kv_lens[i]
    positions (asynchronous on the current stream).  8-bit caches are quantised
    per slot and head.  status: int32[rows] that KV_BAD_* bits are added to."""
    T = _types()
    ca, ra = _cache_args(T, cache), _rows_args(T, rows, k.shape[0])
    code, st, sh = _token_arrays(T, k, v, ca)
    rc = (_lib or lib()).parason_kv_write(ca, ra, k.data_ptr(), v.data_ptr(), code, st, sh,
                                          _status_ptr(T, status, ra.n_rows), _stream(k.device))
    if rc != OK:
        raise ParasonError(rc, "parason_kv_write")


def kv_read(cache: KVCache, rows: KVRows, n_tokens: int, dtype, out=None, status=None):
    """(k, v): the last lengths[i] of row i's kv_lens[i] positions as
    [n_tokens, heads, head_dim] tensors of `dtype` (asynchronous on the current
    stream; `out`: a pair of tensors to write into).  There is no backward pass: a
    cache that requires a gradient is refused while autograd is on."""
    T = _types()
    ca, ra = _cache_args(T, cache), _rows_args(T, rows, int(n_tokens))
    if out is None:
        k, v = out = T.empty((2, int(n_tokens), ca.n_heads, ca.head_dim), dtype=dtype, device=cache.k.device).unbind()
    else:
        k, v = out
    code, st, sh = _token_arrays(T, k, v, ca)
    if k.shape[0] != n_tokens or k.dtype is not dtype:
        raise ValueError("out must hold n_tokens tokens of dtype")
    rc = (_lib or lib()).parason_kv_read(ca, ra, k.data_ptr(), v.data_ptr(), code, st, sh,
                                         _status_ptr(T, status, ra.n_rows), _stream(k.device))
    if rc != OK:
        raise ParasonError(rc, "parason_kv_read")
    return k, v


def tree_attention_workspace_size(cache: KVCache, rows: KVRows, n_tokens: int, q_heads: int) -> int:
    T = _types()
    return _tree_workspace(_cache_args(T, cache), _rows_args(T, rows, int(n_tokens)), int(q_heads))


def _tree_workspace(ca, ra, q_heads: int) -> int:
    b = ctypes.c_size_t()
    rc = (_lib or lib()).parason_tree_attention_workspace_size(ca, ra, q_heads, b)
    if rc != OK:
        raise ParasonError(rc, "parason_tree_attention_workspace_size")
    return b.value


def tree_attention(q, cache: KVCache, rows: KVRows, mask=None, tree_lens=None, scale=None, out=None, lse=False,
                   workspace=None, status=None):
    """Attention of the rows' tokens over the cache (asynchronous on the current
    stream); returns out, or (out, lse).

    q       [tokens, q_heads, head_dim] bfloat16 or float16 (a 16-bit cache's
            own type), any strides with unit stride along a head
    mask    int64 [tokens, words]: the positions of its row's tree that a token
            sees, bit b of word w the position 64 * w + b; None: a chain, where
            every token sees all positions up to its own
    tree_lens  int32 [rows]: the last positions of each row that form its tree
            (default: the row's tokens)
    scale   of the scores (default head_dim ** -0.5)
    lse     True (or a float32 [tokens, q_heads] tensor): also the logarithm of
            each token's and head's sum of exponentials

    There is no backward pass: a q or a cache that requires a gradient is refused
    while autograd is on.
    """
    T = _types()
    code = T.floats.get(q.dtype)
    if code is None or code == DTYPE_F32 or q.dim() != 3 or not q.is_cuda:
        raise TypeError("q must be a [tokens, q_heads, head_dim] bfloat16/float16 device tensor, unit stride along a head")
    if q.requires_grad or (out is not None and out.requires_grad):
        _refuse_gradients(T)
    n_tokens, q_heads, dim = shape = q.shape
    q_st = q.stride()
    if q_st[2] != 1 and dim > 1:
        raise TypeError("q must be a [tokens, q_heads, head_dim] bfloat16/float16 device tensor, unit stride along a head")
    ca, ra = _cache_args(T, cache), _rows_args(T, rows, n_tokens)
    if dim != ca.head_dim:
        raise ValueError("q must have the cache's head_dim")
    if out is None:
        out = T.empty(shape, dtype=q.dtype, device=q.device)
    out_st = out.stride()
    if out.shape != shape or out.dtype is not q.dtype or not out.is_cuda or (out_st[2] != 1 and dim > 1):
        raise TypeError("out must be a device tensor of q's shape and type, unit stride along a head")
    if lse is True:
        lse = T.empty((n_tokens, q_heads), dtype=T.f32, device=q.device)
    elif lse is False:
        lse = None
    elif lse.dtype is not T.f32 or lse.shape != (n_tokens, q_heads) or not lse.is_contiguous() or not lse.is_cuda:
        raise TypeError("lse must be a contiguous float32 [tokens, q_heads] device tensor")
    words = stride = 0
    if mask is not None:
        if mask.dtype is not T.i64 or mask.dim() != 2 or mask.shape[0] != n_tokens or not mask.is_cuda \
                or (mask.stride(1) != 1 and mask.shape[1] > 1):
            raise TypeError("mask must be an int64 [tokens, words] device tensor, unit stride along a token")
        words, stride = mask.shape[1], mask.stride(0)
    if tree_lens is not None and (tree_lens.dtype is not T.i32 or tree_lens.numel() != ra.n_rows
                                  or not tree_lens.is_contiguous() or not tree_lens.is_cuda):
        raise TypeError("tree_lens must be a contiguous int32 device tensor of one entry per row")
    if workspace is None:
        workspace = T.empty(_tree_workspace(ca, ra, q_heads), dtype=T.u8, device=q.device)
    else:
        _check_workspace(T, workspace)
    # (an empty mask has no address, but is one: any address stands for its words, of which none is read)
    mask_ptr = None if mask is None else mask.data_ptr() or workspace.data_ptr()
    ta = TreeArgs(q.data_ptr(), out.data_ptr(), lse.data_ptr() if lse is not None else None, q_st[0], q_st[1],
                  out_st[0], out_st[1], mask_ptr, stride,
                  tree_lens.data_ptr() if tree_lens is not None else None, words, q_heads, code,
                  dim ** -0.5 if scale is None else float(scale))
    rc = (_lib or lib()).parason_tree_attention(ca, ra, ta, _status_ptr(T, status, ra.n_rows), workspace.data_ptr(),
                                                workspace.numel(), _stream(q.device))
    if rc != OK:
        raise ParasonError(rc, "parason_tree_attention")
    return out if lse is None else (out, lse)


@functools.lru_cache(maxsize=256)
def beam_workspace_size(n_groups: int, beams: int, vocab: int) -> int:
    b = ctypes.c_size_t()
    rc = lib().parason_beam_workspace_size(n_groups, beams, vocab, b)
    if rc != OK:
        raise ParasonError(rc, "parason_beam_workspace_size")
    return b.value


def beam_select(logits, scores, beams: int, states=None, workspace=None) -> dict:
    """The `beams` best continuations of every group of `beams` rows
    (asynchronous on the current stream): dict of score (float32), parent (the
    row continued) and token (-1: the row is finished, or the beam empty), int32.

    logits  [rows, vocab] float32/bfloat16/float16, unit stride along the
            vocabulary; -inf forbids a token
    scores  float32 [rows]; -inf: an empty beam
    states  decode states (uint8[rows * 16]) or None: finished rows stay as they
            are, rows with an error are dropped"""
    T = _types()
    code = T.floats.get(logits.dtype)
    if code is None or logits.dim() != 2 or not logits.is_cuda:
        raise TypeError("logits must be a [rows, vocab] float32/bfloat16/float16 device tensor, unit stride")
    rows, vocab = logits.shape
    stride = logits.stride()
    if stride[1] != 1 and vocab > 1:
        raise TypeError("logits must be a [rows, vocab] float32/bfloat16/float16 device tensor, unit stride")
    beams = int(beams)
    if beams < 1 or rows % beams:
        raise ValueError("the rows must be whole groups of beams")
    if scores.dtype is not T.f32 or scores.numel() != rows or not scores.is_contiguous() or not scores.is_cuda:
        raise TypeError("scores must be a contiguous float32 device tensor of one entry per row")
    if states is not None and (states.dtype is not T.u8 or states.numel() != rows * DECODE_STATE_BYTES
                               or not states.is_contiguous() or not states.is_cuda):
        raise TypeError("states must be a contiguous uint8 device tensor of rows * 16 bytes")
    dev = logits.device
    if workspace is None:
        workspace = T.empty(beam_workspace_size(rows // beams, beams, vocab), dtype=T.u8, device=dev)
    else:
        _check_workspace(T, workspace)
    score = scores.new_empty(rows)
    parent, token = T.empty((2, rows), dtype=T.i32, device=dev).unbind()
    rc = (_lib or lib()).parason_beam_select(
        logits.data_ptr(), vocab, stride[0] if rows > 1 else vocab, code, scores.data_ptr(),
        states.data_ptr() if states is not None else None, rows // beams, beams, score.data_ptr(), parent.data_ptr(),
        token.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream(dev))
    if rc != OK:
        raise ParasonError(rc, "parason_beam_select")
    return dict(score=score, parent=parent, token=token)


def beam_reorder(parent, arrays, out=None) -> list:
    """What belongs to the beams, in their new order: row i of every result is
    row parent[i] of the array (asynchronous on the current stream).  arrays: up
    to BEAM_ARRAYS device tensors, each [rows, ...] with contiguous rows, or a
    flat one of rows equal parts; out: tensors to write into, none of whose rows
    lies over these, another's or parent."""
    T = _types()
    rows, n = parent.numel(), len(arrays)
    if parent.dtype is not T.i32 or not parent.is_contiguous() or not parent.is_cuda:
        raise TypeError("parent must be a contiguous int32 device tensor")
    if n > BEAM_ARRAYS:
        raise ValueError("at most %d arrays in one call" % BEAM_ARRAYS)
    if out is not None and len(out) != n:
        raise ValueError("as many results as arrays")
    args, res = (BeamArray * n)(), []
    for i, x in enumerate(arrays):
        if not x.is_cuda:
            raise TypeError("an array must be a device tensor")
        size, stride = _row_bytes(x, rows)
        if out is None:
            y, to = x.new_empty(x.shape), size
        else:
            y = out[i]
            if x.dtype is not y.dtype or x.shape != y.shape or not y.is_cuda:
                raise TypeError("a result must be a device tensor of its array's shape and type")
            to = _row_bytes(y, rows)[1]
        args[i] = (x.data_ptr(), y.data_ptr(), size, stride, to)
        res.append(y)
    rc = (_lib or lib()).parason_beam_reorder(parent.data_ptr(), rows, args, n, _stream(parent.device))
    if rc != OK:
        raise ParasonError(rc, "parason_beam_reorder")
    return res


def _row_bytes(x, rows: int):
    """Bytes of a row of x, and from one row to the next."""
    if x.is_contiguous():
        n = x.numel() * x.element_size()
        if rows == 0 or x.numel() % rows:
            if rows == n == 0:
                return 0, 0
            raise ValueError("an array must have rows equal parts")
        return n // rows, n // rows
    size = x.element_size()
    if x.shape[0] != rows or (rows and not x[0].is_contiguous()) or x.stride(0) < 0:
        raise ValueError("an array must be [rows, ...] with contiguous rows")
    n = x[0].numel() if rows else 0
    return n * size, x.stride(0) * size
