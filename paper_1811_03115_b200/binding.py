"""ctypes binding of libbpd.so: the same calls as include/bpd.h, with argument
marshalling only.  Device buffers come from torch (uint8 tensors); every step
of the decoding path runs inside the library's CUDA kernels.  There is no
fallback: if the library is missing or fails to load, importing this module
raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np

from .build import LIB_PATH


class _Torch:
    """Stands for torch until its first use: sizes, error texts and the raw library need none.  (An import statement in each of the
    operators on a paged cache would cost the smallest of them half a microsecond a call.)"""

    def __getattr__(self, name):
        import torch as module
        globals()["torch"] = module
        return getattr(module, name)


torch = _Torch()

BPD_MAX_K = 16
BPD_OK = 0
STATUS_NAMES = {0: "BPD_OK", -1: "BPD_E_INVALID", -2: "BPD_E_SHAPE", -3: "BPD_E_FORMAT", -4: "BPD_E_NOMEM",
                -5: "BPD_E_STATE", -6: "BPD_E_CUDA", -7: "BPD_E_TIMEOUT", -8: "BPD_E_UNSUPPORTED"}


class BpdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class bpd_stats(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("iterations", C.c_int64), ("invocations", C.c_int64),
                ("row_iterations", C.c_int64), ("khat_hist", C.c_int64 * (BPD_MAX_K + 1)),
                ("device_ms", C.c_double)]


class bpd_iter_out(C.Structure):
    _fields_ = [("khat", C.c_void_p), ("accepted", C.c_void_p), ("table", C.c_void_p),
                ("next_block", C.c_void_p), ("block", C.c_void_p), ("logits_dev", C.c_void_p),
                ("hidden_dev", C.c_void_p), ("layers_dev", C.c_void_p)]


OPTION_FIELDS = ("tensor_cores", "cuda_graphs", "dependent_launch", "lazy_heads", "fold_layer_norms", "cluster_layers",
                 "persistent_layers", "stage_encoder_rows", "l2_stream_hints")


class bpd_session_options(C.Structure):
    _fields_ = [("struct_bytes", C.c_int32)] + [(name, C.c_int32) for name in OPTION_FIELDS]


class bpd_cache(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("page_table", C.c_void_p)] + [
        (name, C.c_int32) for name in ("layers", "n_pages", "pages_per_row", "batch", "kv_heads", "head_dim", "dtype")]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_1811_03115_b200.build "
                      "or __graft_entry__.build()); there is no CPU fallback")
lib = C.CDLL(LIB_PATH)

_vp, _sz, _i, _i64 = C.c_void_p, C.c_size_t, C.c_int, C.c_int64
_SIGS = {
    "bpd_last_error": (C.c_char_p, []),
    "bpd_query_sizes": (_i, [_vp, _sz, _i, _i, _i, C.POINTER(_sz), C.POINTER(_sz)]),
    "bpd_session_bytes": (_i, [_vp, _i, _i, _i, C.POINTER(_sz)]),
    "bpd_session_layer_path": (_i, [_vp]),
    "bpd_load_weights": (_i, [_vp, _sz, _vp, _sz, _vp, C.POINTER(_vp)]),
    "bpd_session_create": (_i, [_vp, _i, _i, _i, _vp, _sz, _vp, C.POINTER(_vp)]),
    "bpd_session_options_init": (None, [C.POINTER(bpd_session_options)]),
    "bpd_session_create_opt": (_i, [_vp, _i, _i, _i, _vp, _sz, _vp, C.POINTER(bpd_session_options), C.POINTER(_vp)]),
    "bpd_session_destroy": (_i, [_vp]),
    "bpd_model_destroy": (_i, [_vp]),
    "bpd_encode": (_i, [_vp, _vp, _vp]),
    "bpd_decode_greedy": (_i, [_vp, _i, C.c_int32, _vp, _vp, C.POINTER(bpd_stats)]),
    "bpd_decode_blockwise": (_i, [_vp, _i, _i, _i, C.c_int32, _vp, _vp, C.POINTER(bpd_stats)]),
    "bpd_decode_blockwise_twocall": (_i, [_vp, _i, _i, _i, C.c_int32, _vp, _vp, C.POINTER(bpd_stats)]),
    "bpd_iteration": (_i, [_vp, _i, _i, _i, C.c_int32, _vp, C.POINTER(bpd_iter_out)]),
    "bpd_set_forced_plan": (_i, [_vp, _vp, _i, _i]),
    "bpd_rewind": (_i, [_vp]),
    "bpd_kernel_launches": (C.c_longlong, []),
    "bpd_profile": (_i, [_vp, _i]),
    "bpd_profile_read": (_i, [_vp, _i, C.POINTER(C.c_int64), C.POINTER(C.c_double)]),
    "bpd_fetch_output": (_i, [_vp, _i, _vp, _vp, C.POINTER(bpd_stats)]),
    "bpd_debug_wait_timeout": (_i, [_vp, _i, _vp]),
    "bpd_op_vocab_argmax_scratch_bytes": (_sz, [_i, _i, _i, _i]),
    "bpd_op_vocab_argmax": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _sz, _vp, _vp, _vp]),
    "bpd_op_vocab_argmax_noalloc": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp]),
    "bpd_op_linear_scratch_bytes": (_sz, [_i, _i, _i, _i]),
    "bpd_op_tree_attention_scratch_bytes": (_sz, [_vp, _i, _i]),
    "bpd_op_tree_attention": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i64, _i64, _vp, _vp, _vp, C.c_float, _vp, _sz, _vp, _vp, _vp]),
    "bpd_op_tree_commit": (_i, [_vp, _vp, _vp, _i, _i64, _vp, _vp, _vp, _vp, _vp, _vp, C.c_int32, _vp, _vp, _vp, _vp, _vp]),
    "bpd_op_cache_weights": (_i, [_vp, _vp, _i, _i, _i64, _vp, _vp, _vp, _vp, _vp, C.c_float, _vp, _vp, _vp]),
    "bpd_op_cache_evict_scratch_bytes": (_sz, [_vp, _i]),
    "bpd_op_cache_evict": (_i, [_vp, _vp, _vp, _i, _i, _vp, _vp, _vp, _sz, _vp, _vp]),
    "bpd_op_page_means": (_i, [_vp, _vp, _vp, _vp, _vp]),
    "bpd_op_page_attention_scratch_bytes": (_sz, [_vp, _i, _i, _i]),
    "bpd_op_page_attention": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i64, _i64, _vp, _vp, _vp, _i, C.c_float, _vp, _sz, _vp, _vp, _vp,
                                   _vp]),
    "bpd_op_status": (_i, [_vp]),
    "bpd_debug_op_wait_timeout": (_i, [_i, _vp]),
    "bpd_op_linear": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _sz, _vp, _vp]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(lib, _name)          # AttributeError here = a declared symbol is not exported
    _fn.restype, _fn.argtypes = _res, _args
EXPORTED = tuple(_SIGS)


def BPD_ACCEPT_TOPN(n: int) -> int:
    return (1 << 8) | (n & 0xff)


def BPD_ACCEPT_DISTANCE(eps: int) -> int:
    return (2 << 8) | (eps & 0xff)


def BPD_ACCEPT_MIN_BLOCK(l: int) -> int:
    return (l & 0xff) << 16


def _check(rc: int) -> None:
    if rc != BPD_OK:
        raise BpdError(rc, lib.bpd_last_error().decode(errors="replace"))


def _host_i32(a, shape=None) -> np.ndarray:
    arr = np.ascontiguousarray(a, dtype=np.int32)
    if shape is not None and tuple(arr.shape) != tuple(shape):
        raise ValueError(f"expected int32 array of shape {shape}, got {arr.shape}")
    return arr


def _ptr(a: Optional[np.ndarray]):
    """Address of an array as the integer a void pointer argument takes (data_as builds a ctypes object: 1.5 us each)."""
    return None if a is None else a.__array_interface__["data"][0]


def _stream() -> int:
    """The current device's current stream (what torch.cuda.current_stream().cuda_stream says, without building the
    stream object: that costs 3 us of a call)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


@dataclass
class Stats:
    tokens: int
    iterations: int
    invocations: int
    row_iterations: int
    khat_hist: list
    device_ms: float

    @property
    def mean_block(self) -> float:
        return self.tokens / max(1, self.row_iterations)


def _stats(st: bpd_stats) -> Stats:
    return Stats(st.tokens, st.iterations, st.invocations, st.row_iterations, list(st.khat_hist), st.device_ms)


def bpd_query_sizes(blob: np.ndarray, batch: int, max_src: int, max_tgt: int):
    wb, sb = _sz(0), _sz(0)
    _check(lib.bpd_query_sizes(_ptr(blob), blob.nbytes, batch, max_src, max_tgt, C.byref(wb), C.byref(sb)))
    return wb.value, sb.value


class Model:
    """bpd_load_weights / bpd_model_destroy.  Owns the torch buffer that holds the weights."""

    def __init__(self, blob: np.ndarray, device: str = "cuda:0"):
        import torch
        blob = np.ascontiguousarray(blob).view(np.uint8)
        wb = _sz(0)
        _check(lib.bpd_query_sizes(_ptr(blob), blob.nbytes, 1, 1, 1, C.byref(wb), None))
        self.device = torch.device(device)
        with torch.cuda.device(self.device):
            self.buf = torch.empty(wb.value, dtype=torch.uint8, device=self.device)
            self.handle = _vp(0)
            _check(lib.bpd_load_weights(_ptr(blob), blob.nbytes, self.buf.data_ptr(), wb.value, _stream(),
                                        C.byref(self.handle)))
        self.blob_header = bytes(blob[:128])

    def close(self):
        if self.handle:
            lib.bpd_model_destroy(self.handle)
            self.handle = _vp(0)


class Session:
    """bpd_session_create_opt and the calls that take a session.  ``options`` maps the field names of
    bpd_session_options to 0 / 1 (anything left out keeps the library's default)."""

    def __init__(self, model: Model, batch: int, max_src: int, max_tgt: int, options: Optional[dict] = None):
        import torch
        opt = bpd_session_options()
        lib.bpd_session_options_init(C.byref(opt))
        for name, value in (options or {}).items():
            if name not in OPTION_FIELDS:
                raise ValueError(f"unknown session option {name!r}")
            setattr(opt, name, int(value))
        self.model, self.B, self.max_src, self.max_tgt = model, batch, max_src, max_tgt
        nb = _sz(0)
        _check(lib.bpd_session_bytes(model.handle, batch, max_src, max_tgt, C.byref(nb)))
        sb = nb.value
        with torch.cuda.device(model.device):
            self.buf = torch.empty(sb, dtype=torch.uint8, device=model.device)
            # a stream of its own: the library replays each decoder pass as a CUDA graph, which the
            # default stream cannot capture.  Time it with events recorded on ``self.stream``.
            self.stream = torch.cuda.Stream(device=model.device)
            self.stream.wait_stream(torch.cuda.current_stream())
            self.handle = _vp(0)
            _check(lib.bpd_session_create_opt(model.handle, batch, max_src, max_tgt, self.buf.data_ptr(), sb,
                                              self.stream.cuda_stream, C.byref(opt), C.byref(self.handle)))
        self.session_bytes = sb

    def close(self):
        if self.handle:
            lib.bpd_session_destroy(self.handle)
            self.handle = _vp(0)

    def bpd_encode(self, src_ids, src_len):
        src = _host_i32(src_ids, (self.B, self.max_src))
        ln = _host_i32(src_len, (self.B,))
        _check(lib.bpd_encode(self.handle, _ptr(src), _ptr(ln)))

    def _decode(self, fn, args, max_new, fetch):
        st = bpd_stats()
        if not fetch:
            _check(fn(self.handle, *args, None, None, None))
            return None
        ids = np.empty((self.B, max_new), dtype=np.int32)
        ln = np.empty(self.B, dtype=np.int32)
        _check(fn(self.handle, *args, _ptr(ids), _ptr(ln), C.byref(st)))
        return ids, ln, _stats(st)

    def bpd_decode_greedy(self, max_new: int, eos_id: int = -1, fetch: bool = True):
        return self._decode(lib.bpd_decode_greedy, (max_new, eos_id), max_new, fetch)

    def bpd_decode_blockwise(self, k: int, max_new: int, eos_id: int = -1, accept_mode: int = 0, fetch: bool = True):
        return self._decode(lib.bpd_decode_blockwise, (k, accept_mode, max_new, eos_id), max_new, fetch)

    def bpd_decode_blockwise_twocall(self, k: int, max_new: int, eos_id: int = -1, accept_mode: int = 0, fetch: bool = True):
        return self._decode(lib.bpd_decode_blockwise_twocall, (k, accept_mode, max_new, eos_id), max_new, fetch)

    def bpd_fetch_output(self, max_new: int):
        st = bpd_stats()
        ids = np.empty((self.B, max_new), dtype=np.int32)
        ln = np.empty(self.B, dtype=np.int32)
        _check(lib.bpd_fetch_output(self.handle, max_new, _ptr(ids), _ptr(ln), C.byref(st)))
        return ids, ln, _stats(st)

    def bpd_rewind(self):
        _check(lib.bpd_rewind(self.handle))

    def bpd_profile(self, enable: bool):
        _check(lib.bpd_profile(self.handle, int(enable)))

    def bpd_profile_read(self, phase: int):
        n, ms = C.c_int64(0), C.c_double(0.0)
        _check(lib.bpd_profile_read(self.handle, phase, C.byref(n), C.byref(ms)))
        return n.value, ms.value

    def bpd_set_forced_plan(self, plan, k: int):
        if plan is None:
            _check(lib.bpd_set_forced_plan(self.handle, None, 0, 0))
            return
        p = _host_i32(plan)
        if p.ndim != 3 or p.shape[0] != self.B or p.shape[2] != k - 1:
            raise ValueError(f"plan must be [batch, plan_len, k-1], got {p.shape}")
        _check(lib.bpd_set_forced_plan(self.handle, _ptr(p), p.shape[1], k))

    def bpd_iteration(self, k: int, max_new: int, eos_id: int = -1, forced_tail=None, accept_mode: int = 0,
                      want_logits: bool = False, want_hidden: bool = False, want_layers: bool = False):
        import torch
        B = self.B
        out = bpd_iter_out()
        khat = np.empty(B, np.int32)
        acc = np.empty((B, k), np.int32)
        table = np.empty((B, k, k), np.int32)
        nxt = np.empty((B, k), np.int32)
        blk = np.empty((B, k), np.int32)
        out.khat, out.accepted, out.table, out.next_block, out.block = (_ptr(khat), _ptr(acc), _ptr(table),
                                                                        _ptr(nxt), _ptr(blk))
        logits = hidden = layers = None
        if want_layers:
            layers = torch.empty((self.n_dec, B, k, self.d_model), dtype=torch.float32, device=self.model.device)
            out.layers_dev = layers.data_ptr()
        if want_logits:
            logits = torch.empty((B, k, k, self.vocab), dtype=torch.float32, device=self.model.device)
            out.logits_dev = logits.data_ptr()
        if want_hidden:
            hidden = torch.empty((B, k, self.d_model), dtype=torch.float32, device=self.model.device)
            out.hidden_dev = hidden.data_ptr()
        tail = None if forced_tail is None else _host_i32(forced_tail, (B, k - 1))
        _check(lib.bpd_iteration(self.handle, k, accept_mode, max_new, eos_id, _ptr(tail), C.byref(out)))
        res = {"khat": khat, "accepted": acc, "table": table, "next_block": nxt, "block": blk}
        if logits is not None:
            res["logits"] = logits
        if hidden is not None:
            res["hidden"] = hidden
        if layers is not None:
            res["layers"] = layers
        return res

    @property
    def layer_path(self) -> int:
        """0: one kernel per projection, 1: three cluster launches per layer, 2: one persistent kernel per pass."""
        return int(lib.bpd_session_layer_path(self.handle))

    @property
    def n_dec(self) -> int:
        return int(np.frombuffer(self.model.blob_header[20:24], np.int32)[0])

    @property
    def vocab(self) -> int:
        return int(np.frombuffer(self.model.blob_header[36:40], np.int32)[0])

    @property
    def d_model(self) -> int:
        return int(np.frombuffer(self.model.blob_header[24:28], np.int32)[0])


def bpd_debug_wait_timeout(limit_us: int = 2000) -> int:
    """Runs the bounded-wait self test and returns the status code (BPD_E_TIMEOUT = -7 is the expected outcome)."""
    import torch
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    return int(lib.bpd_debug_wait_timeout(word.data_ptr(), limit_us, _stream()))


def bpd_kernel_launches() -> int:
    return int(lib.bpd_kernel_launches())


_top1_scratch = {}      # (device, stream) -> scratch tensor, address, bytes: kept from call to call (see _scratch_for)


def _scratch_for(device, stream: int, nbytes: int, captured: bool):
    """A scratch of at least ``nbytes`` for calls on this device and stream.  Calls on one stream run one after the other
    and each leaves the scratch cleared, so they may share it -- also when several threads enqueue on the same stream.
    At most 64 are kept.  A call that is being captured gets a scratch of its own out of the graph's memory: a replay
    comes on any stream and long after the kept one has been replaced."""
    if captured:
        import torch
        t = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return t, t.data_ptr(), nbytes
    key = (device, stream)
    have = _top1_scratch.get(key)
    if have is None or have[2] < nbytes:
        import torch
        if len(_top1_scratch) >= 64:
            _top1_scratch.clear()
        t = torch.empty(nbytes, dtype=torch.uint8, device=device)
        have = _top1_scratch[key] = (t, t.data_ptr(), nbytes)
    return have


def bpd_op_vocab_argmax(x, w, want_val: bool = False):
    """x [rows, d], w [vocab, d]: CUDA tensors, both float32 or both bfloat16.  Returns idx (and val)."""
    import torch
    rows, d = x.shape
    vocab = w.shape[0]
    dtype = 0 if x.dtype == torch.float32 else 1
    device, stream = x.device, _stream()
    # (the bf16 call waits for its result: it cannot be captured)
    scratch = _scratch_for(device, stream, max(lib.bpd_op_vocab_argmax_scratch_bytes(rows, d, vocab, dtype), 256),
                           dtype == 0 and torch.cuda.is_current_stream_capturing())
    idx = torch.empty(rows, dtype=torch.int32, device=device)
    val = torch.empty(rows, dtype=torch.float32, device=device) if want_val else None
    _check(lib.bpd_op_vocab_argmax(x.data_ptr(), w.data_ptr(), rows, d, vocab, dtype, scratch[1], scratch[2],
                                   idx.data_ptr(), None if val is None else val.data_ptr(), stream))
    return (idx, val) if want_val else idx


def bpd_op_vocab_argmax_noalloc(x, w, out_idx, out_val=None):
    """Top-1 of x w^T using the library's built-in workspace: nothing is allocated
    here or in the library, the caller passes the outputs (int32 [rows] and,
    optionally, float32 [rows] CUDA tensors).  For callers that cannot allocate:
    see include/bpd.h for the limits and the sharing rule."""
    import torch
    rows, d = x.shape
    dtype = 0 if x.dtype == torch.float32 else 1
    _check(lib.bpd_op_vocab_argmax_noalloc(x.data_ptr(), w.data_ptr(), rows, d, w.shape[0], dtype,
                                           out_idx.data_ptr(), None if out_val is None else out_val.data_ptr(),
                                           _stream()))


_linear_scratch = {}    # device -> (tensor, address, bytes): bpd_op_linear wants a scratch but never touches it


def bpd_op_linear(x, w, bias=None, relu: bool = False):
    """y = act(x w^T + bias) as float32.  x [rows, in], w [out, in], bias [out] or None."""
    import torch
    rows, in_f = x.shape
    out_f = w.shape[0]
    device = x.device
    y = torch.empty((rows, out_f), dtype=torch.float32, device=device)
    scratch = _linear_scratch.get(device)
    if scratch is None:
        n = lib.bpd_op_linear_scratch_bytes(1, 8, 1, 1)
        t = torch.empty(n, dtype=torch.uint8, device=device)
        scratch = _linear_scratch[device] = (t, t.data_ptr(), n)
    _check(lib.bpd_op_linear(x.data_ptr(), w.data_ptr(), None if bias is None else bias.data_ptr(), rows, in_f, out_f,
                             0 if x.dtype == torch.float32 else 1, int(relu), scratch[1], scratch[2], y.data_ptr(), _stream()))
    return y


# ---------------------------------------------------------------------- operators on a paged cache
# Shapes: pools [layers, pages, 64, kv_heads, head_dim] (one layer's: without the first), page_table int32 [batch,
# pages_per_row], drafted nodes [batch, nodes, heads, head_dim].  float32 or bfloat16 throughout.  All calls enqueue on the
# current stream of the tensors' device and may be captured.  The smallest of them take less time on the device than their
# checks do here, so these are written for speed: the index of a tensor's device instead of the device, one constructor call
# for the structure, no context manager where the device is current already, sizes of new tensors as separate arguments (a
# tuple takes torch twice the time).

def _expect(t, name, shape, dtype, device):
    """Address of a contiguous tensor of this shape and type on the device of this index."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on device {device}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")
    return t.data_ptr()


def _expect_rows(t, name, shape, dtype, device):
    """Address and row stride of a tensor whose last two dimensions are contiguous and whose rows before them are one stride apart."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"{name}: expected a {dtype} tensor of shape {tuple(shape)} on device {device}, got {t.dtype} {tuple(t.shape)} "
                         f"on {t.device}")
    width = shape[-1] * shape[-2]
    if t.is_contiguous():
        return t.data_ptr(), width
    # the stride between rows, and that every dimension in front counts whole groups of rows
    strides, row = t.stride(), None
    ok = (shape[-1] == 1 or strides[-1] == 1) and (shape[-2] == 1 or strides[-2] == shape[-1])
    group = 1
    for n, st in zip(reversed(shape[:-2]), reversed(strides[:-2])):
        if n != 1:
            if row is None:
                row = st
                ok = ok and row >= width
            ok = ok and st == row * group
        group *= n
    if not ok:
        raise ValueError(f"{name}: rows of [heads, head_dim] must be contiguous and one stride apart, got strides {tuple(strides)}")
    return t.data_ptr(), width if row is None else row


def _cache(k_pool, v_pool, page_table, layered: bool):
    """The structure of the calls, and the pool's shape, type and device index."""
    shape, dtype, device = k_pool.shape, k_pool.dtype, k_pool.get_device()
    if len(shape) != (5 if layered else 4) or shape[-3] != 64:
        raise ValueError(f"pools: expected [{'layers, ' if layered else ''}pages, 64, kv_heads, head_dim], got {tuple(shape)}")
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError(f"pools: expected float32 or bfloat16, got {dtype}")
    rows = page_table.shape
    if len(rows) != 2:
        raise ValueError(f"page_table: expected [batch, pages_per_row], got {tuple(rows)}")
    if not k_pool.is_cuda:
        raise ValueError(f"pools: expected CUDA tensors, got {k_pool.device}")
    return bpd_cache(_expect(k_pool, "k_pool", shape, dtype, device), None if v_pool is None else _expect(v_pool, "v_pool", shape, dtype, device),
                     _expect(page_table, "page_table", rows, torch.int32, device), shape[0] if layered else 1, shape[-4], rows[1], rows[0],
                     shape[-2], shape[-1], 0 if dtype is torch.float32 else 1), shape, dtype, device


def _enqueue(device: int, fn, *args):
    """The call on the current stream of this device, with the device current."""
    if torch._C._cuda_getDevice() == device:
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(device))
    if rc != BPD_OK:
        _check(rc)


def _scratch(like, n: int):
    """A tensor of n bytes on a tensor's device, and its address; 0 bytes: none is needed, or the call will refuse its arguments."""
    if n == 0:
        return None, None
    t = like.new_empty(n, dtype=torch.uint8)
    return t, t.data_ptr()


def _drafted(cache, q, k_new, v_new, lens, parents, nodes):
    """Checks of what both attentions take: addresses, sizes and strides in the order of the calls."""
    c, pool, dtype, device = cache
    if q.dim() != 4:
        raise ValueError(f"q: expected [batch, nodes, heads, head_dim], got {tuple(q.shape)}")
    _, t, h, _ = q.shape
    b, hk, d = lens.shape[0] if lens.dim() == 1 else -1, pool[-2], pool[-1]
    if b != c.batch:
        raise ValueError(f"lens: expected [{c.batch}] as the page table has rows, got {tuple(lens.shape)}")
    qp, qs = _expect_rows(q, "q", (b, t, h, d), dtype, device)
    kp, ks = _expect_rows(k_new, "k_new", (b, t, hk, d), dtype, device)
    vp, vs = _expect_rows(v_new, "v_new", (b, t, hk, d), dtype, device)
    if ks != vs:
        raise ValueError(f"k_new and v_new: rows must be the same stride apart, got {ks} and {vs}")
    return (qp, kp, vp, t, h, qs, ks, _expect(lens, "lens", (b,), torch.int32, device), _expect(parents, "parents", (b, t), torch.int32, device),
            None if nodes is None else _expect(nodes, "nodes", (b,), torch.int32, device))


def bpd_op_tree_attention(q, k_new, v_new, k_pool, v_pool, page_table, lens, parents, nodes=None, scale: Optional[float] = None,
                          want_lse: bool = False):
    """Attention of drafted nodes over one layer's cache and their own tree: see include/bpd.h.  q [batch, nodes, heads, head_dim],
    k_new, v_new [batch, nodes, kv_heads, head_dim] (slices of a fused projection will do), lens, nodes int32 [batch], parents
    int32 [batch, nodes].  scale: head_dim ** -0.5 if not given.  Returns out (and lse)."""
    cache = _cache(k_pool, v_pool, page_table, False)
    args = _drafted(cache, q, k_new, v_new, lens, parents, nodes)
    c = C.byref(cache[0])
    n = lib.bpd_op_tree_attention_scratch_bytes(c, args[3], args[4])
    (scratch, at), out = _scratch(q, n), q.new_empty(*q.shape)
    lse = q.new_empty(*q.shape[:3], dtype=torch.float32) if want_lse else None
    _enqueue(cache[3], lib.bpd_op_tree_attention, c, *args, q.shape[3] ** -0.5 if scale is None else scale, at, n, out.data_ptr(),
             lse.data_ptr() if want_lse else None)
    return (out, lse) if want_lse else out


def bpd_op_page_attention(q, k_new, v_new, k_pool, v_pool, page_table, means, lens, parents, select: int, nodes=None,
                          scale: Optional[float] = None, want_lse: bool = False, want_pages: bool = False):
    """bpd_op_tree_attention over the ``select`` best full pages for each node and key head, the open page and the node's line.
    means: float32 [batch, pages_per_row, kv_heads, head_dim].  Returns out, then lse and pages where wanted."""
    cache = _cache(k_pool, v_pool, page_table, False)
    args = _drafted(cache, q, k_new, v_new, lens, parents, nodes)
    (b, per_row), (hk, d), t = page_table.shape, cache[1][-2:], args[3]
    mp = _expect(means, "means", (b, per_row, hk, d), torch.float32, cache[3])
    if select < 1:
        raise ValueError(f"select must be at least 1, got {select}")
    n_sel = min(select, per_row)
    c = C.byref(cache[0])
    n = lib.bpd_op_page_attention_scratch_bytes(c, t, args[4], n_sel)
    (scratch, at), out = _scratch(q, n), q.new_empty(*q.shape)
    lse = q.new_empty(*q.shape[:3], dtype=torch.float32) if want_lse else None
    pages = lens.new_empty(b, t, hk, n_sel) if want_pages else None
    _enqueue(cache[3], lib.bpd_op_page_attention, c, mp, *args, n_sel, d ** -0.5 if scale is None else scale, at, n, out.data_ptr(),
             lse.data_ptr() if want_lse else None, pages.data_ptr() if want_pages else None)
    if want_pages and n_sel < select:
        pages = torch.nn.functional.pad(pages, (0, select - n_sel), value=-1)
    if not want_lse and not want_pages:
        return out
    return (out,) + ((lse,) if want_lse else ()) + ((pages,) if want_pages else ())


def bpd_op_tree_commit(k_new, v_new, k_pool, v_pool, page_table, lens, parents, tokens, top1, last_top1, nodes=None, eos_id: int = -1):
    """Walks every row's tree along the base model's predictions and writes the accepted nodes' keys and values to the caches of
    all layers.  k_new, v_new [layers, batch, nodes, kv_heads, head_dim]; pools with layers.  Returns the new lengths, accepted
    counts, paths [batch, nodes] and the predictions after the paths."""
    c, pool, dtype, device = _cache(k_pool, v_pool, page_table, True)
    if parents.dim() != 2:
        raise ValueError(f"parents: expected [batch, nodes], got {tuple(parents.shape)}")
    b, t, i32 = page_table.shape[0], parents.shape[1], torch.int32
    shape = (pool[0], b, t, pool[3], pool[4])
    kp, ks = _expect_rows(k_new, "k_new", shape, dtype, device)
    vp, vs = _expect_rows(v_new, "v_new", shape, dtype, device)
    if ks != vs:
        raise ValueError(f"k_new and v_new: rows must be the same stride apart, got {ks} and {vs}")
    args = (_expect(lens, "lens", (b,), i32, device), _expect(parents, "parents", (b, t), i32, device), _expect(tokens, "tokens", (b, t), i32, device),
            _expect(top1, "top1", (b, t), i32, device), _expect(last_top1, "last_top1", (b,), i32, device),
            None if nodes is None else _expect(nodes, "nodes", (b,), i32, device))
    new_lens, accepted, following, path = lens.new_empty(b), lens.new_empty(b), lens.new_empty(b), lens.new_empty(b, t)
    _enqueue(device, lib.bpd_op_tree_commit, C.byref(c), kp, vp, t, ks, *args, eos_id, new_lens.data_ptr(), accepted.data_ptr(), path.data_ptr(),
             following.data_ptr())
    return new_lens, accepted, path, following


def bpd_op_cache_weights(q, lse, path, accepted, k_pool, page_table, lens, seen, weights, positions, scale: Optional[float] = None):
    """Adds the attention weights of the accepted nodes to ``weights`` and numbers their own entries in ``positions`` (both
    [batch, kv_heads, capacity], in place).  One layer's pool; ``lens`` are the lengths before the commit."""
    c, pool, dtype, device = _cache(k_pool, None, page_table, False)
    if q.dim() != 4:
        raise ValueError(f"q: expected [batch, nodes, heads, head_dim], got {tuple(q.shape)}")
    (b, per_row), (_, t, h, _), (hk, d), i32 = page_table.shape, q.shape, pool[-2:], torch.int32
    qp, qs = _expect_rows(q, "q", (b, t, h, d), dtype, device)
    state = (b, hk, per_row * 64)
    _enqueue(device, lib.bpd_op_cache_weights, C.byref(c), qp, t, h, qs, _expect(lse, "lse", (b, t, h), torch.float32, device),
             _expect(path, "path", (b, t), i32, device), _expect(accepted, "accepted", (b,), i32, device), _expect(lens, "lens", (b,), i32, device),
             _expect(seen, "seen", (b,), i32, device), d ** -0.5 if scale is None else scale,
             _expect(weights, "weights", state, torch.float32, device), _expect(positions, "positions", state, i32, device))


def bpd_op_cache_evict(weights, positions, k_pool, v_pool, page_table, lens, seen, budget: int, recent: int = 0):
    """Leaves at most ``budget`` entries in every list (layer, row, key head): the last ``recent`` tokens, then the heaviest.
    weights, positions [layers, batch, kv_heads, capacity] and the pools (with layers) change in place.  Returns the new lengths."""
    c, pool, _, device = _cache(k_pool, v_pool, page_table, True)
    (b, per_row), i32 = page_table.shape, torch.int32
    state = (pool[0], b, pool[3], per_row * 64)
    wp, pp = _expect(weights, "weights", state, torch.float32, device), _expect(positions, "positions", state, i32, device)
    lp, sp = _expect(lens, "lens", (b,), i32, device), _expect(seen, "seen", (b,), i32, device)
    ref = C.byref(c)
    n = lib.bpd_op_cache_evict_scratch_bytes(ref, budget)
    (scratch, at), out = _scratch(weights, n), lens.new_empty(b)
    _enqueue(device, lib.bpd_op_cache_evict, ref, lp, sp, budget, recent, wp, pp, at, n, out.data_ptr())
    return out


def bpd_op_page_means(k_pool, page_table, lens_from, lens, means):
    """Means of the keys of the pages that became full between two lengths, into ``means`` float32 [layers, batch, pages_per_row,
    kv_heads, head_dim].  Pool with layers."""
    c, pool, _, device = _cache(k_pool, None, page_table, True)
    b, per_row = page_table.shape
    mp = _expect(means, "means", (pool[0], b, per_row, pool[3], pool[4]), torch.float32, device)
    _enqueue(device, lib.bpd_op_page_means, C.byref(c), _expect(lens_from, "lens_from", (b,), torch.int32, device),
             _expect(lens, "lens", (b,), torch.int32, device), mp)


def bpd_op_status():
    """Raises BpdError (BPD_E_TIMEOUT) if a bounded wait in a kernel of the operators above has expired on the current device since
    the last call.  Synchronises the current stream."""
    _check(lib.bpd_op_status(_stream()))


def bpd_debug_op_wait_timeout(limit_us: int = 2000):
    """Enqueues a wait that expires after about ``limit_us`` microseconds, for bpd_op_status to report once."""
    _check(lib.bpd_debug_op_wait_timeout(limit_us, _stream()))
