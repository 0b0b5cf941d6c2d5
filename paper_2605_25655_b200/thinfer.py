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
# These run once per layer and decode step, so their Python side is kept to plain comparisons: no helper objects, no
# library query for what a few multiplications give.
class _on:
    """Makes the tensors' CUDA device the current one for a call that finds another one current."""

    def __init__(self, device):
        import torch
        self.guard = torch.cuda.device(device)

    def __enter__(self):
        self.guard.__enter__()

    def __exit__(self, *exc):
        self.guard.__exit__(*exc)


class _nothing:
    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_nothing = _nothing()


def _bad(what):
    raise ThinferError(EINVAL, what)


def _enter(device, stream):
    """(guard, raw stream) of a call whose tensors live on `device`: the given stream, or the device's current one."""
    from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice
    if device.type != "cuda":
        _bad(f"tensors must be on a CUDA device, not {device}")
    if stream is None:
        raw = _cuda_getCurrentRawStream(device.index)
    else:
        if stream.device != device:
            _bad(f"the stream belongs to {stream.device}, the tensors to {device}")
        raw = stream.cuda_stream
    return (_nothing if _cuda_getDevice() == device.index else _on(device)), raw


def _ints(t, name, device, shape, dtype=None):
    """Address of a contiguous int32 (or `dtype`) tensor of the given shape."""
    if dtype is None:
        from torch import int32 as dtype
    if t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        _bad(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _token_stride(t, name, dtype, device, shape=None):
    """Elements between the tokens of [tokens, heads, head_dim], whose heads lie side by side."""
    if t.dim() != 3 or t.dtype is not dtype or t.device != device or (shape is not None and t.shape != shape):
        _bad(f"{name}: a {dtype} tensor [tokens, heads, head_dim] on {device}" + (f" of shape {tuple(shape)}" if shape is not None else ""))
    n, h, d = t.shape
    s0, s1, s2 = t.stride()
    if n == 0 or h == 0 or s2 != 1 or (h != 1 and s1 != d):
        _bad(f"{name}: the heads of a token must be contiguous, and there must be some")
    return s0 if n > 1 else h * d


def rope_turns(base, rotary_dim, device="cuda:0"):
    """FP64 [rotary_dim / 2]: revolutions per position of each rotated pair, base^(-2j/rotary_dim) / (2 pi)."""
    import torch
    buf = (C.c_double * max(rotary_dim // 2, 1))()
    _check(lib().thinfer_rope_turns(base, rotary_dim, buf))
    return torch.tensor(list(buf), dtype=torch.float64, device=device)


def op_qk_norm_rope(q, k, q_gain, k_gain, eps, turns, positions, halves=False, q_out=None, k_out=None, stream=None):
    """Per-head RMSNorm and rotation of q [tokens, n_q_heads, d] and k [tokens, n_kv_heads, d] (token strides as they
    come, e.g. slices of a fused projection output); turns from rope_turns (its length sets the rotated dimensions);
    positions int32 [tokens], negative: left as they were.  Returns (q_out, k_out); they may be q and k themselves."""
    import torch
    dev, dt = q.device, q.dtype
    guard, st = _enter(dev, stream)
    qs, ks = _token_stride(q, "q", dt, dev), _token_stride(k, "k", dt, dev)
    n, hq, d = q.shape
    hkv = k.shape[1]
    if k.shape[0] != n or k.shape[2] != d:
        _bad("q and k must agree in tokens and head_dim")
    if q_out is None:
        q_out, qos = torch.empty((n, hq, d), dtype=dt, device=dev), hq * d
    else:
        qos = _token_stride(q_out, "q_out", dt, dev, q.shape)
    if k_out is None:
        k_out, kos = torch.empty((n, hkv, d), dtype=dt, device=dev), hkv * d
    else:
        kos = _token_stride(k_out, "k_out", dt, dev, k.shape)
    if turns.dim() != 1:
        _bad("turns: FP64 [rotary_dim / 2]")
    s = storage_of(q)
    with guard:
        _check(lib(s).thinfer_op_qk_norm_rope(
            q.data_ptr(), qs, k.data_ptr(), ks, q_out.data_ptr(), qos, k_out.data_ptr(), kos, _ints(q_gain, "q_gain", dev, (d,), dt),
            _ints(k_gain, "k_gain", dev, (d,), dt), _ints(turns, "turns", dev, turns.shape, torch.float64),
            _ints(positions, "positions", dev, (n,)), n, hq, hkv, d, 2 * turns.shape[0], int(halves), eps, st), None, s)
    return q_out, k_out


def kv4_page_bytes(n_kv_heads, head_dim, page_size):
    """Bytes of one page of one layer of the 4-bit cache; a pool is a uint8 tensor [n_layers, n_pages, page bytes]."""
    n = C.c_size_t(0)
    _check(lib().thinfer_kv4_page_bytes(n_kv_heads, head_dim, page_size, C.byref(n)))
    return n.value


def _pool(pool, dims, page_size, head_dim, device):
    """Number of KV heads of a uint8 pool tensor whose last dimension is a page."""
    import torch
    if pool.dtype is not torch.uint8 or pool.dim() != dims or not pool.is_contiguous() or pool.device != device:
        _bad(f"pool: a contiguous uint8 tensor of {dims} dimensions on {device}")
    per = page_size * (head_dim + 8)
    heads = pool.shape[-1] // per if per > 0 else 0
    if heads == 0 or heads * per != pool.shape[-1]:
        _bad(f"pool: a page has a multiple of {per} bytes, not {pool.shape[-1]}")
    return heads


def _table(table, device):
    if table.dim() != 2:
        _bad("table: int32 [rows, max_pages]")
    return _ints(table, "table", device, table.shape)


def op_kv4_reserve(table, lens, add, n_pages, page_size, lens_out=None, refused=None, stream=None):
    """Room for add[r] more tokens of every row: writes page numbers into table (int32 [rows, max_pages]); returns
    (lens_out, refused): the new lengths (may be lens itself) and, int64 [1], how many rows did not fit and keep theirs."""
    import torch
    dev = table.device
    guard, st = _enter(dev, stream)
    tab = _table(table, dev)
    rows, max_pages = table.shape
    if lens_out is None:
        lens_out = torch.empty(rows, dtype=torch.int32, device=dev)
    if refused is None:
        refused = torch.empty(1, dtype=torch.int64, device=dev)
    with guard:
        _check(lib().thinfer_op_kv4_reserve(
            tab, _ints(lens, "lens", dev, (rows,)), _ints(add, "add", dev, (rows,)), _ints(lens_out, "lens_out", dev, (rows,)),
            _ints(refused, "refused", dev, (1,), torch.int64), rows, max_pages, n_pages, page_size, st))
    return lens_out, refused


def op_kv4_append(pool, table, k, v, rows, positions, page_size, stream=None):
    """Quantises k, v [tokens, n_kv_heads, d] into one layer's pool [n_pages, page bytes]: token i goes to position
    positions[i] of table row rows[i] (int32 [tokens]; negative: skipped)."""
    dev = pool.device
    guard, st = _enter(dev, stream)
    ks, vs = _token_stride(k, "k", k.dtype, dev), _token_stride(v, "v", k.dtype, dev, k.shape)
    n, hkv, d = k.shape
    if _pool(pool, 2, page_size, d, dev) != hkv:
        _bad("the pool's pages are for another number of heads")
    s = storage_of(k)
    with guard:
        _check(lib(s).thinfer_op_kv4_append(
            pool.data_ptr(), pool.shape[0], _table(table, dev), table.shape[0], table.shape[1], k.data_ptr(), ks, v.data_ptr(), vs,
            _ints(rows, "rows", dev, (n,)), _ints(positions, "positions", dev, (n,)), n, hkv, d, page_size, st), None, s)


def op_kv4_read(pool, table, rows, positions, page_size, head_dim, dtype, k_out=None, v_out=None, stream=None):
    """Values of tokens (rows[i], positions[i]) of one layer: (k, v) [tokens, n_kv_heads, d] of `dtype` (the type the
    pool was written with).  k_out / v_out: two tensors of that shape with equal strides (e.g. transposed views)."""
    import torch
    dev = pool.device
    guard, st = _enter(dev, stream)
    hkv = _pool(pool, 2, page_size, head_dim, dev)
    n = positions.numel()
    shape = (n, hkv, head_dim)
    if k_out is None:
        k_out = torch.empty(shape, dtype=dtype, device=dev)
    if v_out is None:
        v_out = torch.empty_strided(shape, k_out.stride(), dtype=dtype, device=dev)
    strides = k_out.stride()
    for t in (k_out, v_out):
        if t.shape != shape or t.dtype is not dtype or t.device != dev or t.stride() != strides:
            _bad("k_out, v_out: [tokens, heads, head_dim] of one type, device and strides")
    if strides[2] != 1:
        _bad("k_out, v_out: the values of a head must be contiguous")
    s = storage_of(k_out)
    with guard:
        _check(lib(s).thinfer_op_kv4_read(
            pool.data_ptr(), pool.shape[0], _table(table, dev), table.shape[0], table.shape[1], k_out.data_ptr(), v_out.data_ptr(),
            strides[0], strides[1], _ints(rows, "rows", dev, (n,)), _ints(positions, "positions", dev, (n,)), n, hkv, head_dim,
            page_size, st), None, s)
    return k_out, v_out


_workspaces = {}   # sizes -> bytes: what the library answered for them


def op_kv4_attention(q, pool, table, lens, page_size, out=None, workspace=None, stream=None):
    """q [batch, queries, n_q_heads, d] (already rotated) over one layer's 4-bit pool [n_pages, page bytes]: request b is
    row b of table and holds lens[b] keys, the query tokens the last among them.  Returns [batch, queries, n_q_heads, d].
    workspace: uint8, at least thinfer_kv4_attention_workspace bytes (default: allocated for the call)."""
    import torch
    dev, dt = q.device, q.dtype
    guard, st = _enter(dev, stream)
    if q.dim() != 4:
        _bad("q: [batch, queries, n_q_heads, head_dim]")
    b, n, hq, d = q.shape
    s0, s1, s2, s3 = q.stride()
    if b * n * hq == 0 or s3 != 1 or (hq != 1 and s2 != d) or (n > 1 and b > 1 and s0 != n * s1):
        _bad("q: the heads of a token must be contiguous and the query tokens evenly spaced")
    qs = s1 if n > 1 else s0 if b > 1 else hq * d
    hkv = _pool(pool, 2, page_size, d, dev)
    if out is None:
        out = torch.empty((b, n, hq, d), dtype=dt, device=dev)
    s = storage_of(q)
    L = lib(s)
    with guard:
        if workspace is None:
            key = (dev.index, b, n, hq, hkv, d)
            need = _workspaces.get(key)
            if need is None:
                size = C.c_size_t(0)
                _check(L.thinfer_kv4_attention_workspace(b, n, hq, hkv, d, C.byref(size)), None, s)
                need = size.value
                if len(_workspaces) >= 4096:
                    _workspaces.clear()
                _workspaces[key] = need
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        elif workspace.dtype is not torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
            _bad(f"workspace: a contiguous uint8 tensor on {dev}")
        _check(L.thinfer_op_kv4_attention(
            q.data_ptr(), qs, pool.data_ptr(), pool.shape[0], _table(table, dev) if table.shape[0] == b else _bad("table: one row per request"),
            table.shape[1], _ints(lens, "lens", dev, (b,)), _ints(out, "out", dev, (b, n, hq, d), dt), b, n, hq, hkv, d, page_size,
            workspace.data_ptr(), workspace.numel(), st), None, s)
    return out


def _pages_workspace(rows, n_pages, device):
    import torch
    key = (rows, n_pages)
    need = _workspaces.get(key)
    if need is None:
        size = C.c_size_t(0)
        _check(lib().thinfer_kv4_pages_workspace(rows, n_pages, C.byref(size)))
        need = size.value
        if len(_workspaces) >= 4096:
            _workspaces.clear()
        _workspaces[key] = need
    return torch.empty(need, dtype=torch.uint8, device=device)


def op_kv4_fork(pool, table, lens, source, page_size, head_dim, table_out=None, lens_out=None, refused=None, stream=None):
    """New row r takes over old row source[r] (negative: freed) of a pool [n_layers, n_pages, page bytes]: full pages are
    shared, a partly filled last page is copied for every heir but one.  Returns (table_out, lens_out, refused), the last
    int64 [1]."""
    import torch
    dev = pool.device
    guard, st = _enter(dev, stream)
    hkv = _pool(pool, 3, page_size, head_dim, dev)
    tab = _table(table, dev)
    rows, max_pages = table.shape
    if table_out is None:
        table_out = torch.empty((rows, max_pages), dtype=torch.int32, device=dev)
    if lens_out is None:
        lens_out = torch.empty(rows, dtype=torch.int32, device=dev)
    if refused is None:
        refused = torch.empty(1, dtype=torch.int64, device=dev)
    ws = _pages_workspace(rows, pool.shape[1], dev)
    with guard:
        _check(lib().thinfer_op_kv4_fork(
            pool.data_ptr(), pool.shape[0], pool.shape[1], tab, _ints(lens, "lens", dev, (rows,)), _ints(source, "source", dev, (rows,)),
            _ints(table_out, "table_out", dev, (rows, max_pages)), _ints(lens_out, "lens_out", dev, (rows,)),
            _ints(refused, "refused", dev, (1,), torch.int64), rows, max_pages, hkv, head_dim, page_size, ws.data_ptr(), ws.numel(), st))
    return table_out, lens_out, refused


def op_kv4_compact(pool, table, lens, page_size, head_dim, table_out=None, live=None, stream=None):
    """Moves the pages in use of a pool [n_layers, n_pages, page bytes] to its front.  Returns (table_out, live): the table
    with the new page numbers and, int64 [1], the number of pages in use."""
    import torch
    dev = pool.device
    guard, st = _enter(dev, stream)
    hkv = _pool(pool, 3, page_size, head_dim, dev)
    tab = _table(table, dev)
    rows, max_pages = table.shape
    if table_out is None:
        table_out = torch.empty((rows, max_pages), dtype=torch.int32, device=dev)
    if live is None:
        live = torch.empty(1, dtype=torch.int64, device=dev)
    ws = _pages_workspace(rows, pool.shape[1], dev)
    with guard:
        _check(lib().thinfer_op_kv4_compact(
            pool.data_ptr(), pool.shape[0], pool.shape[1], tab, _ints(lens, "lens", dev, (rows,)),
            _ints(table_out, "table_out", dev, (rows, max_pages)), _ints(live, "live", dev, (1,), torch.int64), rows, max_pages, hkv,
            head_dim, page_size, ws.data_ptr(), ws.numel(), st))
    return table_out, live


def to_device_layers(np_layers, device="cuda:0"):
    """numpy FP16 weight dicts (synth.layer_weights) -> torch CUDA tensors."""
    import torch
    return [{k: torch.from_numpy(v).to(device) for k, v in w.items()} for w in np_layers]
