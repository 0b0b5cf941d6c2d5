"""ctypes binding over libthinfer.so (include/thinfer.h).

Argument marshalling only: torch supplies device memory and streams, every step
of the path runs in the library's CUDA kernels.  There is no CPU fallback: if
the shared library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libthinfer.so")
# one build per 16-bit storage type, same exports (include/thinfer.h)
LIB_PATHS = {"f16": LIB_PATH, "bf16": os.path.join(_HERE, "libthinfer_bf16.so")}

OK, EINVAL, EUNSUPPORTED, ECAPACITY, EBUSY, ECUDA, ETIMEOUT = 0, -1, -2, -3, -4, -5, -6
ERR_NAMES = {OK: "THINFER_OK", EINVAL: "THINFER_EINVAL", EUNSUPPORTED: "THINFER_EUNSUPPORTED",
             ECAPACITY: "THINFER_ECAPACITY", EBUSY: "THINFER_EBUSY", ECUDA: "THINFER_ECUDA",
             ETIMEOUT: "THINFER_ETIMEOUT"}
K_RMSNORM, K_QKV, K_ATTN, K_ATTN_COMBINE, K_OPROJ, K_GATEUP, K_DOWN, K_HEAD, K_EMBED, K_ARGMAX, K_DECODE_UNIFIED = range(11)

EXPORTS = (
    "thinfer_storage_type", "thinfer_workspace_bytes", "thinfer_create", "thinfer_prefill", "thinfer_prefill_ragged", "thinfer_slot_lengths",
    "thinfer_decode_step",
    "thinfer_prefill_host", "thinfer_decode_step_host", "thinfer_release_slot", "thinfer_slot_state",
    "thinfer_kv_pointer", "thinfer_status", "thinfer_clear_status", "thinfer_capture_hidden", "thinfer_set_launch_mode", "thinfer_profile_select",
    "thinfer_profile_read", "thinfer_trace_unified", "thinfer_launch_count", "thinfer_last_error", "thinfer_destroy",
    "thinfer_op_linear", "thinfer_op_linear_noalloc", "thinfer_op_attention_prefill", "thinfer_op_rmsnorm",
    "thinfer_op_argmax", "thinfer_op_attention_decode", "thinfer_selftest_bounded_wait",
    "thinfer_rope_turns", "thinfer_op_qk_norm_rope", "thinfer_kv4_page_bytes", "thinfer_op_kv4_reserve",
    "thinfer_op_kv4_append", "thinfer_op_kv4_read", "thinfer_kv4_attention_workspace", "thinfer_op_kv4_attention",
    "thinfer_kv4_pages_workspace", "thinfer_op_kv4_fork", "thinfer_op_kv4_compact",
)


class ThinferError(RuntimeError):
    def __init__(self, code, what=""):
        self.code = code
        super().__init__(f"{ERR_NAMES.get(code, code)}: {what}")


class Config(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("ffn", C.c_int32), ("n_layers", C.c_int32), ("vocab", C.c_int32),
                ("rms_eps", C.c_float), ("rope_base", C.c_float), ("max_batch", C.c_int32),
                ("max_seq", C.c_int32), ("buf_slots", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class Weights(C.Structure):
    _fields_ = [("layers", C.POINTER(LayerWeights)), ("embed", C.c_void_p), ("final_norm", C.c_void_p),
                ("lm_head", C.c_void_p)]


_libs = {}


def storage_of(tensor) -> str:
    """'f16' or 'bf16' for a torch tensor of a storage type the library is built for."""
    import torch
    if tensor.dtype == torch.float16:
        return "f16"
    if tensor.dtype == torch.bfloat16:
        return "bf16"
    raise ThinferError(EUNSUPPORTED, f"storage type {tensor.dtype}: the library is built for float16 and bfloat16")


def lib(storage="f16"):
    """Loads the shared library of a storage type (once).  Fails loudly when it has not been built."""
    if storage in _libs:
        return _libs[storage]
    path = LIB_PATHS[storage]
    if not os.path.exists(path):
        raise ThinferError(ECUDA, f"{path} is missing: build it with "
                                  "`python -m paper_2605_25655_b200._build` (needs nvcc)")
    L = C.CDLL(path)
    L.thinfer_storage_type.argtypes = []
    assert L.thinfer_storage_type() == {"f16": 0, "bf16": 1}[storage], path
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    L.thinfer_workspace_bytes.argtypes = [C.POINTER(Config), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    L.thinfer_create.argtypes = [C.POINTER(Config), C.POINTER(Weights), vp, C.c_size_t, vp, C.c_size_t, C.POINTER(vp)]
    L.thinfer_prefill.argtypes = [vp, i32, vp, i32, i32, vp, vp, vp]
    L.thinfer_prefill_ragged.argtypes = [vp, i32, vp, i32, i32, C.POINTER(i32), vp, vp, vp]
    L.thinfer_slot_lengths.argtypes = [vp, i32, C.POINTER(i32)]
    L.thinfer_decode_step.argtypes = [vp, i32, vp, vp, vp, vp]
    L.thinfer_prefill_host.argtypes = [vp, i32, vp, i32, i32, vp, vp, vp]
    L.thinfer_decode_step_host.argtypes = [vp, i32, vp, vp, vp, vp]
    L.thinfer_release_slot.argtypes = [vp, i32, vp]
    L.thinfer_slot_state.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(i32)]
    L.thinfer_kv_pointer.argtypes = [vp, i32, i32, i32, C.POINTER(vp)]
    L.thinfer_status.argtypes = [vp, C.POINTER(i32)]
    L.thinfer_clear_status.argtypes = [vp]
    L.thinfer_capture_hidden.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(vp)]
    L.thinfer_set_launch_mode.argtypes = [vp, i32]
    L.thinfer_profile_select.argtypes = [vp, i32]
    L.thinfer_profile_read.argtypes = [vp, C.POINTER(i32), C.POINTER(C.c_float)]
    L.thinfer_trace_unified.argtypes = [vp, i32, C.POINTER(C.c_uint64), i32]
    L.thinfer_launch_count.argtypes = [vp]
    L.thinfer_launch_count.restype = i64
    L.thinfer_last_error.argtypes = [vp]
    L.thinfer_last_error.restype = C.c_char_p
    L.thinfer_destroy.argtypes = [vp]
    L.thinfer_destroy.restype = None
    L.thinfer_op_linear.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp]
    L.thinfer_op_linear_noalloc.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp]
    L.thinfer_op_attention_prefill.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp]
    L.thinfer_op_rmsnorm.argtypes = [vp, vp, vp, i32, i32, C.c_float, vp]
    L.thinfer_op_argmax.argtypes = [vp, vp, i32, i32, vp]
    L.thinfer_op_attention_decode.argtypes = [vp, i32, i32, vp, vp, i32, i32, C.POINTER(i32), vp]
    L.thinfer_selftest_bounded_wait.argtypes = [vp, i64, vp]
    szp = C.POINTER(C.c_size_t)
    L.thinfer_rope_turns.argtypes = [C.c_float, i32, C.POINTER(C.c_double)]
    L.thinfer_op_qk_norm_rope.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32,
                                          C.c_float, vp]
    L.thinfer_kv4_page_bytes.argtypes = [i32, i32, i32, szp]
    L.thinfer_op_kv4_reserve.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, vp]
    L.thinfer_op_kv4_append.argtypes = [vp, i32, vp, i32, i32, vp, i64, vp, i64, vp, vp, i32, i32, i32, i32, vp]
    L.thinfer_op_kv4_read.argtypes = [vp, i32, vp, i32, i32, vp, vp, i64, i64, vp, vp, i32, i32, i32, i32, vp]
    L.thinfer_kv4_attention_workspace.argtypes = [i32, i32, i32, i32, i32, szp]
    L.thinfer_op_kv4_attention.argtypes = [vp, i64, vp, i32, vp, i32, vp, vp, i32, i32, i32, i32, i32, i32, vp, C.c_size_t, vp]
    L.thinfer_kv4_pages_workspace.argtypes = [i32, i32, szp]
    L.thinfer_op_kv4_fork.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, C.c_size_t, vp]
    L.thinfer_op_kv4_compact.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, C.c_size_t, vp]
    _libs[storage] = L
    return L


def _check(rc, ctx=None, storage="f16"):
    if rc != OK:
        msg = lib(storage).thinfer_last_error(ctx)
        raise ThinferError(rc, msg.decode() if msg else "")


def _stream_ptr(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def make_config(shape, max_batch, max_seq, buf_slots=1) -> Config:
    """shape: any object with the fields of synth.Shape."""
    return Config(shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn, shape.n_layers,
                  shape.vocab, shape.rms_eps, shape.rope_base, max_batch, max_seq, buf_slots)


def workspace_bytes(cfg: Config, storage="f16"):
    kv, sc = C.c_size_t(0), C.c_size_t(0)
    _check(lib(storage).thinfer_workspace_bytes(C.byref(cfg), C.byref(kv), C.byref(sc)), None, storage)
    return kv.value, sc.value


class Context:
    """One thinfer_ctx plus the torch tensors that back its caller-owned memory.

    layers: list of dicts name -> CUDA float16 (or bfloat16) tensor (names of thinfer_layer_weights);
    stack:  dict with embed / final_norm / lm_head when shape.vocab > 0.
    """

    def __init__(self, shape, layers, stack=None, max_batch=1, max_seq=128, buf_slots=1, device="cuda:0"):
        import torch
        self.torch = torch
        self.shape = shape
        self.device = torch.device(device)
        self.cfg = make_config(shape, max_batch, max_seq, buf_slots)
        self.storage = storage_of(layers[0]["wq"])         # the weights decide which build serves this context
        self.dtype = layers[0]["wq"].dtype
        self.L = lib(self.storage)
        kv_bytes, scratch_bytes = workspace_bytes(self.cfg, self.storage)
        with torch.cuda.device(self.device):
            self.kv = torch.empty(kv_bytes, dtype=torch.uint8, device=self.device)
            self.scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=self.device)
            self._keep = (layers, stack)
            arr = (LayerWeights * shape.n_layers)()
            for l, w in enumerate(layers):
                for name, _ in LayerWeights._fields_:
                    t = w[name]
                    assert t.is_cuda and t.dtype == self.dtype and t.is_contiguous(), name
                    setattr(arr[l], name, t.data_ptr())
            wts = Weights(arr, None, None, None)
            if shape.vocab > 0:
                wts.embed, wts.final_norm, wts.lm_head = (stack[n].data_ptr() for n in ("embed", "final_norm", "lm_head"))
            h = C.c_void_p(None)
            _check(self.L.thinfer_create(C.byref(self.cfg), C.byref(wts), self.kv.data_ptr(), kv_bytes,
                                         self.scratch.data_ptr(), scratch_bytes, C.byref(h)), None, self.storage)
        self.h = h

    # -- device-buffer calls ------------------------------------------------
    def prefill(self, inp, slot=0, stream=None, want_logits=False, out=None):
        torch = self.torch
        batch, seq = int(inp.shape[0]), int(inp.shape[1])
        assert inp.is_cuda and inp.is_contiguous()
        if self.shape.vocab == 0:
            assert inp.dtype == self.dtype
            out = torch.empty_like(inp)
            _check(self.L.thinfer_prefill(self.h, slot, inp.data_ptr(), batch, seq, out.data_ptr(), None,
                                         _stream_ptr(stream)), self.h, self.storage)
            return out
        assert inp.dtype == torch.int32
        ids = torch.empty(batch, dtype=torch.int32, device=self.device) if out is None else out
        logits = torch.empty(batch, self.shape.vocab, dtype=torch.float32, device=self.device) if want_logits else None
        _check(self.L.thinfer_prefill(self.h, slot, inp.data_ptr(), batch, seq, ids.data_ptr(),
                                     logits.data_ptr() if want_logits else None, _stream_ptr(stream)), self.h, self.storage)
        return (ids, logits) if want_logits else ids

    def prefill_ragged(self, inp, seq_lens, slot=0, stream=None, want_logits=False):
        """Prompts of different lengths, padded to inp.shape[1]; seq_lens: one length per request."""
        torch = self.torch
        batch, seq = int(inp.shape[0]), int(inp.shape[1])
        lens = (C.c_int32 * batch)(*[int(v) for v in seq_lens])
        assert inp.is_cuda and inp.is_contiguous()
        if self.shape.vocab == 0:
            out = torch.empty_like(inp)
            _check(self.L.thinfer_prefill_ragged(self.h, slot, inp.data_ptr(), batch, seq, lens, out.data_ptr(), None,
                                                _stream_ptr(stream)), self.h, self.storage)
            return out
        ids = torch.empty(batch, dtype=torch.int32, device=self.device)
        logits = torch.empty(batch, self.shape.vocab, dtype=torch.float32, device=self.device) if want_logits else None
        _check(self.L.thinfer_prefill_ragged(self.h, slot, inp.data_ptr(), batch, seq, lens, ids.data_ptr(),
                                            logits.data_ptr() if want_logits else None, _stream_ptr(stream)), self.h, self.storage)
        return (ids, logits) if want_logits else ids

    def slot_lengths(self, slot=0):
        b, _ = self.slot_state(slot)
        buf = (C.c_int32 * max(b, 1))()
        _check(self.L.thinfer_slot_lengths(self.h, slot, buf), self.h, self.storage)
        return list(buf)[:b]

    def decode_step(self, inp, slot=0, stream=None, want_logits=False, out=None):
        torch = self.torch
        assert inp.is_cuda and inp.is_contiguous()
        if self.shape.vocab == 0:
            out = torch.empty_like(inp) if out is None else out
            _check(self.L.thinfer_decode_step(self.h, slot, inp.data_ptr(), out.data_ptr(), None,
                                             _stream_ptr(stream)), self.h, self.storage)
            return out
        batch = int(inp.shape[0])
        ids = torch.empty(batch, dtype=torch.int32, device=self.device) if out is None else out
        logits = torch.empty(batch, self.shape.vocab, dtype=torch.float32, device=self.device) if want_logits else None
        _check(self.L.thinfer_decode_step(self.h, slot, inp.data_ptr(), ids.data_ptr(),
                                         logits.data_ptr() if want_logits else None, _stream_ptr(stream)), self.h, self.storage)
        return (ids, logits) if want_logits else ids

    # -- host-buffer calls (pinned tensors make the copies asynchronous) -----
    def prefill_host(self, host_in, host_out, slot=0, stream=None, host_logits=None):
        batch, seq = int(host_in.shape[0]), int(host_in.shape[1])
        _check(self.L.thinfer_prefill_host(self.h, slot, host_in.data_ptr(), batch, seq, host_out.data_ptr(),
                                          host_logits.data_ptr() if host_logits is not None else None,
                                          _stream_ptr(stream)), self.h, self.storage)

    def decode_step_host(self, host_in, host_out, slot=0, stream=None, host_logits=None):
        _check(self.L.thinfer_decode_step_host(self.h, slot, host_in.data_ptr(), host_out.data_ptr(),
                                              host_logits.data_ptr() if host_logits is not None else None,
                                              _stream_ptr(stream)), self.h, self.storage)

    # -- bookkeeping ----------------------------------------------------------
    def release_slot(self, slot=0, stream=None):
        _check(self.L.thinfer_release_slot(self.h, slot, _stream_ptr(stream)), self.h, self.storage)

    def slot_state(self, slot=0):
        b, n = C.c_int32(0), C.c_int32(0)
        _check(self.L.thinfer_slot_state(self.h, slot, C.byref(b), C.byref(n)), self.h, self.storage)
        return b.value, n.value

    def kv_view(self, slot, layer, which):
        """Strided torch view [max_batch][n_kv_heads][max_seq][head_dim] of K (0) or V (1)."""
        p = C.c_void_p(None)
        _check(self.L.thinfer_kv_pointer(self.h, slot, layer, which, C.byref(p)), self.h, self.storage)
        off = p.value - self.kv.data_ptr()
        n = self.cfg.max_batch * self.cfg.n_kv_heads * self.cfg.max_seq * self.cfg.head_dim
        return self.kv[off:off + 2 * n].view(self.dtype).view(
            self.cfg.max_batch, self.cfg.n_kv_heads, self.cfg.max_seq, self.cfg.head_dim)

    def status(self):
        v = C.c_int32(0)
        _check(self.L.thinfer_status(self.h, C.byref(v)), self.h, self.storage)
        return v.value

    def clear_status(self):
        _check(self.L.thinfer_clear_status(self.h), self.h, self.storage)

    def attention_decode(self, q, t_len, slot=0, layer=0, seq_lens=None, stream=None):
        """Decode attention alone over the cache of (slot, layer): q [batch, n_q_heads, head_dim] -> [batch, n_q_heads*d]."""
        batch = int(q.shape[0])
        out = self.torch.empty(batch, self.shape.n_q_heads * self.shape.head_dim, dtype=q.dtype, device=q.device)
        lens = (C.c_int32 * batch)(*[int(v) for v in seq_lens]) if seq_lens is not None else None
        _check(self.L.thinfer_op_attention_decode(self.h, slot, layer, q.data_ptr(), out.data_ptr(), batch, int(t_len),
                                                  lens, _stream_ptr(stream)), self.h, self.storage)
        return out

    def selftest_bounded_wait(self, limit_ns=1_000_000, stream=None):
        _check(self.L.thinfer_selftest_bounded_wait(self.h, int(limit_ns), _stream_ptr(stream)), self.h, self.storage)

    def capture_hidden(self, captures):
        """captures: dict layer index (-1 = input of layer 0) -> CUDA FP16 tensor that receives the hidden
        state behind that layer on every later prefill / decode step; {} or None removes all captures."""
        captures = captures or {}
        n = len(captures)
        layers = (C.c_int32 * max(n, 1))(*[int(l) for l in captures])
        bufs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in captures.values()])
        self._captures = captures                      # keeps the tensors alive
        _check(self.L.thinfer_capture_hidden(self.h, n, layers, bufs), self.h, self.storage)

    def set_launch_mode(self, mode):
        _check(self.L.thinfer_set_launch_mode(self.h, mode), self.h, self.storage)

    def profile_select(self, kernel_id):
        _check(self.L.thinfer_profile_select(self.h, kernel_id), self.h, self.storage)

    def profile_read(self):
        n, ms = C.c_int32(0), C.c_float(0)
        _check(self.L.thinfer_profile_read(self.h, C.byref(n), C.byref(ms)), self.h, self.storage)
        return n.value, ms.value

    def trace_unified(self, enable=True, read=0):
        """Switches the unit-boundary trace of the unified decode kernel on/off; returns `read` entries (ns)."""
        buf = (C.c_uint64 * max(read, 1))()
        _check(self.L.thinfer_trace_unified(self.h, int(enable), buf if read else None, read), self.h, self.storage)
        return list(buf)[:read]

    def launch_count(self):
        return int(self.L.thinfer_launch_count(self.h))

    def close(self):
        if self.h is not None and self.h.value:
            self.L.thinfer_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- operators
def op_linear(x, w, out_fp32=False, path=0, stream=None, out=None):
    import torch
    rows, k = x.shape
    n_out = w.shape[0]
    if out is not None:
        y, out_fp32 = out, out.dtype == torch.float32
    else:
        y = torch.empty(rows, n_out, dtype=torch.float32 if out_fp32 else x.dtype, device=x.device)
    st = storage_of(x)
    _check(lib(st).thinfer_op_linear(x.data_ptr(), w.data_ptr(), y.data_ptr(), rows, n_out, k, int(out_fp32), path,
                                     _stream_ptr(stream)), None, st)
    return y


def op_linear_noalloc(x, w, y, stream=None):
    """y[rows, n_out] = x w^T through the entry point that allocates nothing: the caller passes
    the output (FP16 or FP32 tensor); the split-K scratch is a fixed array inside the library.
    For hosts that cannot call cudaMalloc where they need the product.  rows <= 16, n_out <= 16384."""
    import torch
    rows, k = x.shape
    n_out = w.shape[0]
    assert y.shape == (rows, n_out) and y.is_contiguous()
    st = storage_of(x)
    _check(lib(st).thinfer_op_linear_noalloc(x.data_ptr(), w.data_ptr(), y.data_ptr(), rows, n_out, k,
                                             int(y.dtype == torch.float32), _stream_ptr(stream)), None, st)
    return y


def op_attention_prefill(q, k, v, seq=None, stream=None, out=None):
    """q [B, Hq, S, d]; k, v [B, Hkv, T, d] with T >= S (the first S positions are used) -> [B, S, Hq*d]."""
    import torch
    b, hq, s, d = q.shape
    hkv, t = k.shape[1], k.shape[2]
    if out is None:
        out = torch.empty(b, s, hq * d, dtype=q.dtype, device=q.device)
    st = storage_of(q)
    _check(lib(st).thinfer_op_attention_prefill(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), b, hq, hkv,
                                                s, t, d, _stream_ptr(stream)), None, st)
    return out


def op_rmsnorm(x, gain, eps, stream=None):
    import torch
    rows, n = x.shape
    y = torch.empty_like(x)
    st = storage_of(x)
    _check(lib(st).thinfer_op_rmsnorm(x.data_ptr(), gain.data_ptr(), y.data_ptr(), rows, n, eps, _stream_ptr(stream)), None, st)
    return y


def op_argmax(logits, stream=None):
    import torch
    rows, n = logits.shape
    ids = torch.empty(rows, dtype=torch.int32, device=logits.device)
    _check(lib().thinfer_op_argmax(logits.data_ptr(), ids.data_ptr(), rows, n, _stream_ptr(stream)))
    return ids


# ------------------------------------- per-head norm + rotation, 4-bit paged cache
class _On:
    """Checks that tensors live on one CUDA device and makes it the current one for the call; hands out its stream."""

    def __init__(self, device, stream=None):
        import torch
        if device.type != "cuda":
            raise ThinferError(EINVAL, f"tensors must be on a CUDA device, not {device}")
        self.device, self.torch = device, torch
        if stream is not None and stream.device != device:
            raise ThinferError(EINVAL, f"the stream belongs to {stream.device}, the tensors to {device}")
        self.guard = None if torch.cuda.current_device() == device.index else torch.cuda.device(device)
        self.stream = stream

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        s = self.stream if self.stream is not None else self.torch.cuda.current_stream(self.device)
        return s.cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _want(ok, what):
    if not ok:
        raise ThinferError(EINVAL, what)


def _want_int32(device, **tensors):
    import torch
    for name, (t, shape) in tensors.items():
        _want(t.dtype == torch.int32 and t.device == device and t.is_contiguous() and tuple(t.shape) == tuple(shape),
              f"{name}: a contiguous int32 tensor of shape {tuple(shape)} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _token_stride(t, name, dtype, device):
    """Elements between the tokens of [tokens, heads, head_dim], whose heads lie side by side."""
    _want(t.dim() == 3 and t.dtype == dtype and t.device == device, f"{name}: [tokens, heads, head_dim] {dtype} on {device}")
    n, h, d = t.shape
    _want(n > 0 and h > 0 and t.stride(2) == 1 and (h == 1 or t.stride(1) == d), f"{name}: the heads of a token must be contiguous")
    return t.stride(0) if n > 1 else -(-max(t.stride(0), h * d) // 8) * 8


def rope_turns(base, rotary_dim, device="cuda:0"):
    """FP64 [rotary_dim / 2]: revolutions per position of each rotated pair, base^(-2j/rotary_dim) / (2 pi)."""
    import torch
    buf = (C.c_double * (rotary_dim // 2))()
    _check(lib().thinfer_rope_turns(base, rotary_dim, buf))
    return torch.tensor(list(buf), dtype=torch.float64, device=device)


def op_qk_norm_rope(q, k, q_gain, k_gain, eps, turns, positions, halves=False, q_out=None, k_out=None, stream=None):
    """Per-head RMSNorm and rotation of q [tokens, n_q_heads, d] and k [tokens, n_kv_heads, d] (token strides as they
    come, e.g. slices of a fused projection output); turns from rope_turns (its length sets the rotated dimensions);
    positions int32 [tokens], negative: left as they were.  Returns (q_out, k_out); they may be q and k themselves."""
    import torch
    dev = q.device
    with _On(dev, stream) as st:
        n, hq, d = q.shape if q.dim() == 3 else (0, 0, 0)
        qs, ks = _token_stride(q, "q", q.dtype, dev), _token_stride(k, "k", q.dtype, dev)
        hkv = k.shape[1]
        _want(k.shape[0] == n and k.shape[2] == d, "q and k must agree in tokens and head_dim")
        for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
            _want(g.dtype == q.dtype and g.device == dev and g.is_contiguous() and tuple(g.shape) == (d,), f"{name}: [head_dim] {q.dtype} on {dev}")
        _want(turns.dtype == torch.float64 and turns.device == dev and turns.is_contiguous() and turns.dim() == 1, "turns: FP64 [rotary_dim / 2]")
        _want_int32(dev, positions=(positions, (n,)))
        q_out = torch.empty(n, hq, d, dtype=q.dtype, device=dev) if q_out is None else q_out
        k_out = torch.empty(n, hkv, d, dtype=q.dtype, device=dev) if k_out is None else k_out
        _want(tuple(q_out.shape) == (n, hq, d) and tuple(k_out.shape) == (n, hkv, d), "q_out / k_out: the shapes of q / k")
        qos, kos = _token_stride(q_out, "q_out", q.dtype, dev), _token_stride(k_out, "k_out", q.dtype, dev)
        s = storage_of(q)
        _check(lib(s).thinfer_op_qk_norm_rope(q.data_ptr(), qs, k.data_ptr(), ks, q_out.data_ptr(), qos, k_out.data_ptr(), kos,
                                              q_gain.data_ptr(), k_gain.data_ptr(), turns.data_ptr(), positions.data_ptr(), n, hq,
                                              hkv, d, 2 * turns.shape[0], int(halves), eps, st), None, s)
    return q_out, k_out


def kv4_page_bytes(n_kv_heads, head_dim, page_size):
    """Bytes of one page of one layer of the 4-bit cache; a pool is a uint8 tensor [n_layers, n_pages, page bytes]."""
    n = C.c_size_t(0)
    _check(lib().thinfer_kv4_page_bytes(n_kv_heads, head_dim, page_size, C.byref(n)))
    return n.value


def _pool(pool, dims, page_size, head_dim):
    """Number of KV heads of a uint8 pool tensor whose last dimension is a page."""
    import torch
    _want(pool.dtype == torch.uint8 and pool.dim() == dims and pool.is_contiguous(), f"pool: a contiguous uint8 tensor of {dims} dimensions")
    per = kv4_page_bytes(1, head_dim, page_size)
    _want(pool.shape[-1] > 0 and pool.shape[-1] % per == 0, f"pool: a page has a multiple of {per} bytes, not {pool.shape[-1]}")
    return pool.shape[-1] // per


def op_kv4_reserve(table, lens, add, n_pages, page_size, lens_out=None, refused=None, stream=None):
    """Room for add[r] more tokens of every row: writes page numbers into table (int32 [rows, max_pages]); returns
    (lens_out, refused): the new lengths and how many rows did not fit (they keep their length)."""
    import torch
    dev = table.device
    with _On(dev, stream) as st:
        rows, max_pages = table.shape
        lens_out = torch.empty_like(lens) if lens_out is None else lens_out
        refused = torch.empty(1, dtype=torch.int32, device=dev) if refused is None else refused
        _want_int32(dev, table=(table, (rows, max_pages)), lens=(lens, (rows,)), add=(add, (rows,)), lens_out=(lens_out, (rows,)),
                    refused=(refused, (1,)))
        _check(lib().thinfer_op_kv4_reserve(table.data_ptr(), lens.data_ptr(), add.data_ptr(), lens_out.data_ptr(), refused.data_ptr(),
                                            rows, max_pages, n_pages, page_size, st))
    return lens_out, refused


def op_kv4_append(pool, table, k, v, rows, positions, page_size, stream=None):
    """Quantises k, v [tokens, n_kv_heads, d] into one layer's pool [n_pages, page bytes]: token i goes to position
    positions[i] of table row rows[i] (int32 [tokens]; negative: skipped)."""
    dev = pool.device
    with _On(dev, stream) as st:
        ks, vs = _token_stride(k, "k", k.dtype, dev), _token_stride(v, "v", k.dtype, dev)
        n, hkv, d = k.shape
        _want(tuple(v.shape) == (n, hkv, d), "k and v must have one shape")
        _want(_pool(pool, 2, page_size, d) == hkv, "the pool's pages are for another number of heads")
        _want_int32(dev, table=(table, table.shape), rows=(rows, (n,)), positions=(positions, (n,)))
        _want(table.dim() == 2, "table: [rows, max_pages]")
        s = storage_of(k)
        _check(lib(s).thinfer_op_kv4_append(pool.data_ptr(), pool.shape[0], table.data_ptr(), table.shape[0], table.shape[1],
                                            k.data_ptr(), ks, v.data_ptr(), vs, rows.data_ptr(), positions.data_ptr(), n, hkv, d,
                                            page_size, st), None, s)


def op_kv4_read(pool, table, rows, positions, page_size, head_dim, dtype, k_out=None, v_out=None, stream=None):
    """Values of tokens (rows[i], positions[i]) of one layer: (k, v) [tokens, n_kv_heads, d] of `dtype` (the type the
    pool was written with).  k_out / v_out: two tensors of that shape with equal strides (e.g. transposed views)."""
    import torch
    dev = pool.device
    with _On(dev, stream) as st:
        hkv = _pool(pool, 2, page_size, head_dim)
        n = positions.shape[0]
        k_out = torch.empty(n, hkv, head_dim, dtype=dtype, device=dev) if k_out is None else k_out
        v_out = torch.empty(n, hkv, head_dim, dtype=dtype, device=dev) if v_out is None else v_out
        for t in (k_out, v_out):
            _want(tuple(t.shape) == (n, hkv, head_dim) and t.dtype == dtype and t.device == dev and t.stride(2) == 1 and
                  t.stride() == k_out.stride(), "k_out, v_out: [tokens, heads, head_dim], equal strides")
        _want(table.dim() == 2, "table: [rows, max_pages]")
        _want_int32(dev, table=(table, table.shape), rows=(rows, (n,)), positions=(positions, (n,)))
        s = storage_of(k_out)
        _check(lib(s).thinfer_op_kv4_read(pool.data_ptr(), pool.shape[0], table.data_ptr(), table.shape[0], table.shape[1],
                                          k_out.data_ptr(), v_out.data_ptr(), k_out.stride(0), k_out.stride(1), rows.data_ptr(),
                                          positions.data_ptr(), n, hkv, head_dim, page_size, st), None, s)
    return k_out, v_out


def op_kv4_attention(q, pool, table, lens, page_size, out=None, workspace=None, stream=None):
    """q [batch, queries, n_q_heads, d] (already rotated) over one layer's 4-bit pool [n_pages, page bytes]: request b is
    row b of table and holds lens[b] keys, the query tokens the last among them.  Returns [batch, queries, n_q_heads, d]."""
    import torch
    dev = q.device
    with _On(dev, stream) as st:
        _want(q.dim() == 4, "q: [batch, queries, n_q_heads, head_dim]")
        b, n, hq, d = q.shape
        _want(b == 1 or n == 1 or q.stride(0) == n * q.stride(1), "q: the query tokens must be evenly spaced")
        flat = q.reshape(b * n, hq, d) if n == 1 or q.is_contiguous() else q.view(b * n, hq, d)
        qs = _token_stride(flat, "q", q.dtype, dev)
        hkv = _pool(pool, 2, page_size, d)
        _want(pool.device == dev, f"pool: on {dev}")
        _want(table.dim() == 2, "table: [batch, max_pages]")
        _want_int32(dev, table=(table, (b, table.shape[1])), lens=(lens, (b,)))
        out = torch.empty(b, n, hq, d, dtype=q.dtype, device=dev) if out is None else out
        _want(tuple(out.shape) == (b, n, hq, d) and out.dtype == q.dtype and out.device == dev and out.is_contiguous(), "out: contiguous, the shape of q")
        s = storage_of(q)
        L = lib(s)
        if workspace is None:
            need = C.c_size_t(0)
            _check(L.thinfer_kv4_attention_workspace(b, n, hq, hkv, d, C.byref(need)), None, s)
            workspace = torch.empty(need.value, dtype=torch.uint8, device=dev)
        _check(L.thinfer_op_kv4_attention(flat.data_ptr(), qs, pool.data_ptr(), pool.shape[0], table.data_ptr(), table.shape[1],
                                          lens.data_ptr(), out.data_ptr(), b, n, hq, hkv, d, page_size, workspace.data_ptr(),
                                          workspace.numel() * workspace.element_size(), st), None, s)
    return out


def _pages_workspace(rows, n_pages, device):
    import torch
    need = C.c_size_t(0)
    _check(lib().thinfer_kv4_pages_workspace(rows, n_pages, C.byref(need)))
    return torch.empty(need.value, dtype=torch.uint8, device=device)


def op_kv4_fork(pool, table, lens, source, page_size, head_dim, table_out=None, lens_out=None, refused=None, stream=None):
    """New row r takes over old row source[r] (negative: freed) of a pool [n_layers, n_pages, page bytes]: full pages are
    shared, a partly filled last page is copied for every heir but one.  Returns (table_out, lens_out, refused)."""
    import torch
    dev = pool.device
    with _On(dev, stream) as st:
        hkv = _pool(pool, 3, page_size, head_dim)
        _want(table.dim() == 2, "table: [rows, max_pages]")
        rows, max_pages = table.shape
        table_out = torch.empty_like(table) if table_out is None else table_out
        lens_out = torch.empty_like(lens) if lens_out is None else lens_out
        refused = torch.empty(1, dtype=torch.int32, device=dev) if refused is None else refused
        _want_int32(dev, table=(table, (rows, max_pages)), lens=(lens, (rows,)), source=(source, (rows,)),
                    table_out=(table_out, (rows, max_pages)), lens_out=(lens_out, (rows,)), refused=(refused, (1,)))
        ws = _pages_workspace(rows, pool.shape[1], dev)
        _check(lib().thinfer_op_kv4_fork(pool.data_ptr(), pool.shape[0], pool.shape[1], table.data_ptr(), lens.data_ptr(),
                                         source.data_ptr(), table_out.data_ptr(), lens_out.data_ptr(), refused.data_ptr(), rows,
                                         max_pages, hkv, head_dim, page_size, ws.data_ptr(), ws.numel(), st))
    return table_out, lens_out, refused


def op_kv4_compact(pool, table, lens, page_size, head_dim, table_out=None, live=None, stream=None):
    """Moves the pages in use of a pool [n_layers, n_pages, page bytes] to its front.  Returns (table_out, live): the table
    with the new page numbers and the number of pages in use."""
    import torch
    dev = pool.device
    with _On(dev, stream) as st:
        hkv = _pool(pool, 3, page_size, head_dim)
        _want(table.dim() == 2, "table: [rows, max_pages]")
        rows, max_pages = table.shape
        table_out = torch.empty_like(table) if table_out is None else table_out
        live = torch.empty(1, dtype=torch.int32, device=dev) if live is None else live
        _want_int32(dev, table=(table, (rows, max_pages)), lens=(lens, (rows,)), table_out=(table_out, (rows, max_pages)), live=(live, (1,)))
        ws = _pages_workspace(rows, pool.shape[1], dev)
        _check(lib().thinfer_op_kv4_compact(pool.data_ptr(), pool.shape[0], pool.shape[1], table.data_ptr(), lens.data_ptr(),
                                            table_out.data_ptr(), live.data_ptr(), rows, max_pages, hkv, head_dim, page_size,
                                            ws.data_ptr(), ws.numel(), st))
    return table_out, live


def to_device_layers(np_layers, device="cuda:0"):
    """numpy FP16 weight dicts (synth.layer_weights) -> torch CUDA tensors."""
    import torch
    return [{k: torch.from_numpy(v).to(device) for k, v in w.items()} for w in np_layers]
