"""Thin ctypes binding of libtts_gpt.so: same names as the C ABI, argument marshalling only.

PyTorch is used for device memory and streams; every step of the decode path runs inside the
library's CUDA kernels.  If the shared library is missing or fails to load, ``load()`` raises:
there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os

import numpy as np
import torch

from .cases import GPTConfig, LINEARS, W_BF16

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtts_gpt.so")

OK, E_ARG, E_NO_PAGES, E_STREAM, E_CTX_OVERFLOW, E_CUDA, E_TIMEOUT, E_WORKSPACE, E_UNSUPPORTED = \
    0, -1, -2, -3, -4, -5, -6, -7, -8

EXPORTS = [
    "tts_gpt_query_workspace", "tts_gpt_create", "tts_gpt_prefill", "tts_gpt_prefill_tokens", "tts_gpt_decode_step", "tts_gpt_decode_step_host", "tts_gpt_decode_steps",
    "tts_gpt_release_stream", "tts_gpt_sync", "tts_gpt_destroy", "tts_gpt_last_error",
    "tts_gpt_stats", "tts_gpt_stream_context", "tts_gpt_debug_shuffle_free_pages",
    "tts_gpt_debug_kernel_launches", "tts_gpt_debug_set_trace", "tts_gpt_debug_expire_wait", "tts_gpt_debug_expire_linear", "tts_gpt_debug_expire_op", "tts_gpt_debug_set_option", "tts_gpt_debug_check_canaries",
    "tts_gpt_op_linear_packed_bytes", "tts_gpt_op_linear_pack", "tts_gpt_op_linear",
    "tts_gpt_op_linear_tc_scratch_bytes", "tts_gpt_op_linear_tc", "tts_gpt_op_attention_scratch_bytes", "tts_gpt_op_attention", "tts_gpt_op_attention_static", "tts_gpt_op_attention_cluster",
    "tts_gpt_op_layernorm",
    "tts_gpt_op_sample",
    "tts_gpt_op_page_tables", "tts_gpt_op_kv_append", "tts_gpt_op_attention_shared_scratch_bytes", "tts_gpt_op_attention_shared",
    "tts_gpt_op_attention_cross_scratch_bytes", "tts_gpt_op_attention_cross",
    "tts_gpt_op_rope_frequencies", "tts_gpt_op_rope_kv_append", "tts_gpt_op_tree_tables", "tts_gpt_op_attention_tree_scratch_bytes", "tts_gpt_op_attention_tree",
    "tts_gpt_op_tree_accept", "tts_gpt_op_kv_move",
]
T_F32, T_BF16, T_F16 = 0, 1, 2
_TYPES = {torch.float32: T_F32, torch.bfloat16: T_BF16, torch.int16: T_BF16, torch.float16: T_F16}   # int16: bf16 bits
# Argument types of the calls below that are made once a step or more: declared, ctypes converts plain numbers itself, several
# times faster than from objects made for each argument.
_i, _l, _p, _f, _d = C.c_int32, C.c_int64, C.c_void_p, C.c_float, C.c_double  # noqa: E741
_ARGTYPES = {
    "tts_gpt_op_page_tables": [_i, _p, _p, _i, _p, _p, _i, _p, _p, _p, _i, _p, _i, _p, _i, _p, _p, _p, _p, _p, _p],
    "tts_gpt_op_kv_append": [_i, _i, _i, _p, _l, _p, _l, _p, _i, _i, _p, _p],
    "tts_gpt_op_attention_shared": [_i, _i, _i, _i, _p, _l, _i, _i, _p, _i, _p, _i, _p, _p, _p, _p, C.c_size_t, _p],
    "tts_gpt_op_attention_cross": [_i, _i, _i, _i, _i, _p, _l, _i, _p, _l, _l, _p, _l, _l, _p, _p, _i, C.c_float, _p, _p, C.c_size_t, _p],
    "tts_gpt_op_rope_frequencies": [_i, _i, _d, _d, _d, _d, _d, _p, _p, _p],
    "tts_gpt_op_rope_kv_append": [_i, _i, _i, _i, _p, _l, _p, _l, _p, _l, _p, _p, _i, _p, _i, _f, _i, _p, _l, _i, _i, _p, _p],
    "tts_gpt_op_tree_tables": [_i, _i, _p, _p, _i, _p, _p, _i, _p, _p, _p, _p],
    "tts_gpt_op_attention_tree": [_i, _i, _i, _i, _i, _p, _l, _i, _i, _p, _i, _p, _i, _p, _p, _p, _i, _p, _i, _f, _p, _p, C.c_size_t, _p],
    "tts_gpt_op_tree_accept": [_i, _i, _p, _p, _p, _p, _p, _i, _p, _p, _p, _i, _i, _p, _p, _p, _p, _p, _p, _p, _p],
    "tts_gpt_op_kv_move": [_i, _i, _p, _p, _p, _i, _i, _i, _i, _l, _p, _p],
}


class TtsGptError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("tts_gpt error %d: %s" % (code, msg))
        self.code = code


class ConfigStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layer", "d_model", "n_head", "head_dim", "d_ff", "vocab", "wfmt", "max_streams",
                 "max_context", "page_tokens", "n_pages", "max_pos", "gelu_tanh", "stop_token")] + \
               [("ln_eps", C.c_float), ("emb_rows", C.c_int32), ("kv_fmt", C.c_int32)]


_PP = C.POINTER(C.c_void_p)


class WeightsStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("tok_emb", "pos_emb", "lnf_g", "lnf_b", "head_w", "head_b")] + \
               [(n, _PP) for n in ("ln1_g", "ln1_b", "ln2_g", "ln2_b",
                                   "qkv_w", "qkv_s", "qkv_b", "o_w", "o_s", "o_b",
                                   "fc1_w", "fc1_s", "fc1_b", "fc2_w", "fc2_s", "fc2_b")]


_lib = None


def load() -> C.CDLL:
    """Open the shared library (once).  Raises OSError if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError("%s not found: build it with `python -m paper_2607_21042_b200.build` "
                          "(no CPU fallback exists)" % LIB_PATH)
        lib = C.CDLL(LIB_PATH)
        lib.tts_gpt_last_error.restype = C.c_char_p
        lib.tts_gpt_last_error.argtypes = [C.c_void_p]
        for name in EXPORTS:
            if name != "tts_gpt_last_error":
                getattr(lib, name).restype = C.c_int32
        for name, types in _ARGTYPES.items():
            getattr(lib, name).argtypes = types
        _lib = lib
    return _lib


def _check(rc, handle=None):
    if rc != OK:
        msg = load().tts_gpt_last_error(handle)
        raise TtsGptError(rc, msg.decode() if msg else "")
    return rc


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    if isinstance(t, torch.Tensor):
        return C.c_void_p(t.data_ptr())
    return C.c_void_p(int(t))


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _i32_array(vals):
    return (C.c_int32 * len(vals))(*[int(v) for v in vals])


def to_device_bits(arr, device):
    """numpy array of bf16 bit patterns (uint16), int8 codes or int32 words -> device tensor."""
    if arr is None:
        return None
    if isinstance(arr, torch.Tensor):
        return arr.to(device)
    a = np.ascontiguousarray(arr)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    return torch.from_numpy(a).to(device)


def config_struct(cfg: GPTConfig) -> ConfigStruct:
    return ConfigStruct(**cfg.as_dict())


def query_workspace(cfg: GPTConfig) -> int:
    n = C.c_size_t(0)
    cs = config_struct(cfg)
    _check(load().tts_gpt_query_workspace(C.byref(cs), C.byref(n)))
    return n.value


class TtsGpt:
    """One engine on one GPU.  Methods mirror the C entry points."""

    def __init__(self, cfg: GPTConfig, weights: dict, device="cuda:0", stream=None):
        self.lib = load()
        self.cfg = cfg
        self.device = torch.device(device)
        self.handle = None
        torch.cuda.set_device(self.device)
        # The engine enqueues on a stream of its own (a non-default stream, so that the step can be
        # captured into a CUDA graph).  Work the caller queued on torch's current stream is ordered
        # before the engine's by `wait_for_caller()`, which prefill calls; decode_step does not (its
        # inputs are normally produced long before), so synchronise or call it yourself when a
        # buffer handed to decode_step was written on another stream just before.
        self.stream = stream if stream is not None else torch.cuda.Stream(self.device)
        dev_w = {}
        for k, v in weights.items():
            if isinstance(v, list):
                dev_w[k] = [to_device_bits(x, self.device) for x in v]
            else:
                dev_w[k] = to_device_bits(v, self.device)
        ws = WeightsStruct()
        keep = []
        for name in ("tok_emb", "pos_emb", "lnf_g", "lnf_b", "head_w", "head_b"):
            setattr(ws, name, _ptr(dev_w.get(name)).value)
        per_layer = ["ln1_g", "ln1_b", "ln2_g", "ln2_b"] + [l + s for l in LINEARS for s in ("_w", "_s", "_b")]
        for name in per_layer:
            ptrs = [(_ptr(t).value or 0) for t in dev_w[name]]
            arr = (C.c_void_p * len(ptrs))(*ptrs)
            keep.append(arr)
            setattr(ws, name, C.cast(arr, _PP))
        nbytes = query_workspace(cfg)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        cs = config_struct(cfg)
        h = C.c_void_p(0)
        torch.cuda.synchronize(self.device)
        _check(self.lib.tts_gpt_create(C.byref(cs), C.byref(ws), C.c_void_p(base), C.c_size_t(nbytes),
                                       C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self.handle = h
        self.workspace_bytes = nbytes
        del dev_w, keep

    def wait_for_caller(self):
        """Order everything queued so far on torch's current stream before the engine's next work."""
        self.stream.wait_stream(torch.cuda.current_stream(self.device))

    # -- the five calls -----------------------------------------------------------------------
    def prefill(self, prefixes, top_k=0, temperature=1.0, uniforms=None, pos0=None,
                out_tokens=None, out_logits=None, out_hidden=None):
        """prefixes: list of device tensors (int16 view of bf16 bits or torch.bfloat16) [P_i, d].
        Returns (stream_ids list, out_tokens tensor)."""
        n = len(prefixes)
        self.wait_for_caller()
        self._live_prefixes = [p.contiguous() for p in prefixes]
        ptrs = (C.c_void_p * n)(*[p.data_ptr() for p in self._live_prefixes])
        lens = _i32_array([p.shape[0] for p in self._live_prefixes])
        ids = (C.c_int32 * n)()
        if out_tokens is None:
            out_tokens = torch.empty(n, dtype=torch.int32, device=self.device)
        p0 = _i32_array(pos0) if pos0 is not None else None
        _check(self.lib.tts_gpt_prefill(self.handle, C.c_int32(n), ptrs, lens, p0, C.c_int32(top_k),
                                        C.c_float(temperature), _ptr(uniforms), ids, _ptr(out_tokens),
                                        _ptr(out_logits), _ptr(out_hidden)), self.handle)
        return list(ids), out_tokens

    def prefill_tokens(self, cond, text_ids, text_shift, text_pos0, top_k=0, temperature=1.0, uniforms=None,
                       pos0=None, out_tokens=None, out_logits=None, out_hidden=None):
        """Prefixes assembled on the device: cond[i] a device tensor of bf16 bits [n_cond_i, d] (or None),
        text_ids[i] a device int32 tensor [n_text_i] (or None).  Returns (stream_ids list, out_tokens tensor)."""
        n = len(cond)
        self.wait_for_caller()
        self._live_prefixes = [None if p is None else p.contiguous() for p in cond]
        self._live_text = [None if t is None else t.contiguous() for t in text_ids]
        cptrs = (C.c_void_p * n)(*[None if p is None else p.data_ptr() for p in self._live_prefixes])
        tptrs = (C.c_void_p * n)(*[None if t is None else t.data_ptr() for t in self._live_text])
        ncond = _i32_array([0 if p is None else p.shape[0] for p in self._live_prefixes])
        ntext = _i32_array([0 if t is None else t.shape[0] for t in self._live_text])
        ids = (C.c_int32 * n)()
        if out_tokens is None:
            out_tokens = torch.empty(n, dtype=torch.int32, device=self.device)
        p0 = _i32_array(pos0) if pos0 is not None else None
        _check(self.lib.tts_gpt_prefill_tokens(self.handle, C.c_int32(n), cptrs, ncond, tptrs, ntext,
                                               C.c_int32(text_shift), C.c_int32(text_pos0), p0, C.c_int32(top_k),
                                               C.c_float(temperature), _ptr(uniforms), ids, _ptr(out_tokens),
                                               _ptr(out_logits), _ptr(out_hidden)), self.handle)
        return list(ids), out_tokens

    def decode_step(self, stream_ids, out_tokens, in_tokens=None, top_k=0, temperature=1.0,
                    uniforms=None, out_logits=None, out_hidden=None):
        n = len(stream_ids)
        ids = stream_ids if isinstance(stream_ids, C.Array) else _i32_array(stream_ids)
        return _check(self.lib.tts_gpt_decode_step(self.handle, C.c_int32(n), ids, _ptr(in_tokens),
                                                   C.c_int32(top_k), C.c_float(temperature),
                                                   _ptr(uniforms), _ptr(out_tokens), _ptr(out_logits),
                                                   _ptr(out_hidden)), self.handle)

    def decode_step_host(self, stream_ids, out_tokens, in_tokens=None, top_k=0, temperature=1.0,
                         uniforms=None, out_logits=None, out_hidden=None):
        """One step with HOST tensors (ideally pinned): inputs are copied in, results are valid on return."""
        n = len(stream_ids)
        ids = stream_ids if isinstance(stream_ids, C.Array) else _i32_array(stream_ids)
        return _check(self.lib.tts_gpt_decode_step_host(self.handle, C.c_int32(n), ids, _ptr(in_tokens),
                                                        C.c_int32(top_k), C.c_float(temperature),
                                                        _ptr(uniforms), _ptr(out_tokens), _ptr(out_logits),
                                                        _ptr(out_hidden)), self.handle)

    def decode_steps(self, stream_ids, n_steps, out_tokens, in_tokens=None, top_k=0, temperature=1.0,
                     uniforms=None, out_logits=None, out_hidden=None):
        """n_steps steps in one call; the output tensors hold n_steps * len(stream_ids) rows."""
        n = len(stream_ids)
        ids = stream_ids if isinstance(stream_ids, C.Array) else _i32_array(stream_ids)
        return _check(self.lib.tts_gpt_decode_steps(self.handle, C.c_int32(n), ids, _ptr(in_tokens),
                                                    C.c_int32(n_steps), C.c_int32(top_k), C.c_float(temperature),
                                                    _ptr(uniforms), _ptr(out_tokens), _ptr(out_logits),
                                                    _ptr(out_hidden)), self.handle)

    def release_stream(self, stream_id):
        return _check(self.lib.tts_gpt_release_stream(self.handle, C.c_int32(stream_id)), self.handle)

    def sync(self):
        rc = _check(self.lib.tts_gpt_sync(self.handle), self.handle)
        self._live_prefixes = None
        return rc

    def destroy(self):
        if self.handle is not None:
            self.lib.tts_gpt_destroy(self.handle)
            self.handle = None
            self.workspace = None

    # -- introspection ------------------------------------------------------------------------
    def stats(self):
        a, b = C.c_int32(0), C.c_int32(0)
        _check(self.lib.tts_gpt_stats(self.handle, C.byref(a), C.byref(b)), self.handle)
        return {"open_streams": a.value, "free_pages": b.value}

    def stream_context(self, stream_id):
        return int(self.lib.tts_gpt_stream_context(self.handle, C.c_int32(stream_id)))

    def kernel_launches(self):
        n = C.c_uint64(0)
        _check(self.lib.tts_gpt_debug_kernel_launches(self.handle, C.byref(n)), self.handle)
        return n.value

    def set_trace(self, trace_tensor):
        """trace_tensor: int64 device tensor with 8 * slots entries (or None to switch off).
        Returns the number of traced kernels per step."""
        n = C.c_int32(0)
        _check(self.lib.tts_gpt_debug_set_trace(self.handle, _ptr(trace_tensor), C.byref(n)), self.handle)
        return n.value

    def debug_shuffle_free_pages(self, seed):
        return _check(self.lib.tts_gpt_debug_shuffle_free_pages(self.handle, C.c_uint32(seed)), self.handle)

    def set_option(self, name, value):
        """Switch a kernel schedule on or off, or set a threshold (see tts_gpt_debug_set_option)."""
        return _check(self.lib.tts_gpt_debug_set_option(self.handle, C.c_char_p(name.encode()), C.c_int32(int(value))),
                      self.handle)

    def check_canaries(self):
        """Number of guard bytes around the KV pool that were overwritten (0 = intact)."""
        n = C.c_int32(0)
        _check(self.lib.tts_gpt_debug_check_canaries(self.handle, C.byref(n)), self.handle)
        return n.value

    def debug_expire_wait(self, limit_us):
        return _check(self.lib.tts_gpt_debug_expire_wait(self.handle, C.c_uint32(limit_us)), self.handle)

    def debug_expire_linear(self, kernel, rows, tile, limit_us, out):
        return _check(self.lib.tts_gpt_debug_expire_linear(self.handle, C.c_int32(kernel), C.c_int32(rows), C.c_int32(tile),
                                                           C.c_uint32(limit_us), _ptr(out)), self.handle)

    def raw_call(self, name, *args):
        """Return the raw status of a C entry point (tests of error behaviour)."""
        return getattr(self.lib, name)(self.handle, *args)

    def last_error(self):
        m = self.lib.tts_gpt_last_error(self.handle)
        return m.decode() if m else ""

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---------------------------------------------------------------------------------------------
# single-kernel entry points
# ---------------------------------------------------------------------------------------------
def op_linear_pack(wfmt, w, s, stream=None):
    """w: device tensor in the canonical format [N,K] (bf16 bits int16 / int8 / int32 words
    [N,K/8]); s: scales or None.  Returns the packed device buffer."""
    lib = load()
    N = w.shape[0]
    K = w.shape[1] * (8 if wfmt == 2 else 1)
    nbytes = C.c_size_t(0)
    _check(lib.tts_gpt_op_linear_packed_bytes(C.c_int32(wfmt), C.c_int32(N), C.c_int32(K), C.byref(nbytes)))
    packed = torch.empty(nbytes.value, dtype=torch.uint8, device=w.device)
    assert packed.data_ptr() % 256 == 0
    _check(lib.tts_gpt_op_linear_pack(C.c_int32(wfmt), C.c_int32(N), C.c_int32(K), _ptr(w), _ptr(s),
                                      _ptr(packed), _stream_ptr(stream)))
    return packed, N, K


def op_linear(wfmt, packed, N, K, act, bias=None, stream=None):
    B = act.shape[0]
    out = torch.empty((B, N), dtype=torch.float32, device=act.device)
    _check(load().tts_gpt_op_linear(C.c_int32(wfmt), C.c_int32(N), C.c_int32(K), _ptr(packed), _ptr(bias),
                                    C.c_int32(B), _ptr(act), _ptr(out), _stream_ptr(stream)))
    return out


def op_linear_tc(wfmt, w, s, act, bias=None, ksplit=1, stream=None):
    """Tensor-core linear: w/s in the canonical formats, act int16 (bf16 bits) [B,K] -> fp32 [B,N]."""
    N = w.shape[0]
    K = w.shape[1] * (8 if wfmt == 2 else 1)
    B = act.shape[0]
    n = C.c_size_t(0)
    _check(load().tts_gpt_op_linear_tc_scratch_bytes(C.c_int32(N), C.c_int32(K), C.byref(n)))
    scratch = torch.zeros(n.value + 1024, dtype=torch.uint8, device=w.device)
    base = (scratch.data_ptr() + 1023) // 1024 * 1024
    out = torch.empty((B, N), dtype=torch.float32, device=w.device)
    _check(load().tts_gpt_op_linear_tc(C.c_int32(wfmt), C.c_int32(N), C.c_int32(K), _ptr(w), _ptr(s), _ptr(bias),
                                       C.c_int32(B), _ptr(act), _ptr(out), C.c_int32(ksplit), C.c_void_p(base),
                                       _stream_ptr(stream)))
    (torch.cuda.current_stream() if stream is None else stream).synchronize()
    del scratch
    return out


def op_attention_scratch(R, n_head, device):
    n = C.c_size_t(0)
    _check(load().tts_gpt_op_attention_scratch_bytes(C.c_int32(R), C.c_int32(n_head), C.byref(n)))
    return torch.zeros(n.value, dtype=torch.uint8, device=device)


def op_attention(q, kv_layer, page_table, row_stream, row_pos, scratch=None, stream=None):
    R, dm = q.shape
    H = dm // 64
    out = torch.empty((R, dm), dtype=torch.int16, device=q.device)
    if scratch is None:
        scratch = op_attention_scratch(R, H, q.device)
    _check(load().tts_gpt_op_attention(C.c_int32(R), C.c_int32(H), _ptr(q), _ptr(kv_layer), _ptr(page_table),
                                       C.c_int32(page_table.shape[1]), _ptr(row_stream), _ptr(row_pos),
                                       _ptr(out), _ptr(scratch), _stream_ptr(stream)))
    return out


def op_attention_cluster(q, kv_layer, page_table, row_stream, row_pos, cluster_size, stream=None):
    """cluster_size 1, 2, 4, 8: cluster variant; 0: streaming variant; -1: prefill variant on the CUDA cores,
    -2: prefill variant on the tensor cores (both: rows grouped by stream with ascending positions)."""
    R, dm = q.shape
    H = dm // 64
    out = torch.empty((R, dm), dtype=torch.int16, device=q.device)
    _check(load().tts_gpt_op_attention_cluster(C.c_int32(R), C.c_int32(H), _ptr(q), _ptr(kv_layer),
                                               _ptr(page_table), C.c_int32(page_table.shape[1]),
                                               _ptr(row_stream), _ptr(row_pos), _ptr(out),
                                               C.c_int32(cluster_size), _stream_ptr(stream)))
    return out


STATIC_ATTN_MAX_ROW_HEADS = 1280


def op_attention_static(q, kv_layer, page_table, row_stream, row_pos, stream=None):
    """Attention for callers that may not allocate: scratch is an array inside the library (at most
    STATIC_ATTN_MAX_ROW_HEADS rows x heads).  Only the output tensor is created here, by torch; pass
    your own through the C entry point to avoid even that.  Calls on one device must not overlap."""
    R, dm = q.shape
    H = dm // 64
    out = torch.empty((R, dm), dtype=torch.int16, device=q.device)
    _check(load().tts_gpt_op_attention_static(C.c_int32(R), C.c_int32(H), _ptr(q), _ptr(kv_layer),
                                              _ptr(page_table), C.c_int32(page_table.shape[1]),
                                              _ptr(row_stream), _ptr(row_pos), _ptr(out), _stream_ptr(stream)))
    return out


def op_layernorm(x, g, b, eps, stream=None):
    R, d = x.shape
    out = torch.empty((R, d), dtype=torch.int16, device=x.device)
    _check(load().tts_gpt_op_layernorm(C.c_int32(R), C.c_int32(d), _ptr(x), _ptr(g), _ptr(b), C.c_float(eps),
                                       _ptr(out), _stream_ptr(stream)))
    return out


def op_sample(logits, top_k=0, temperature=1.0, uniforms=None, stream=None):
    R, V = logits.shape
    out = torch.empty(R, dtype=torch.int32, device=logits.device)
    _check(load().tts_gpt_op_sample(C.c_int32(R), C.c_int32(V), _ptr(logits), C.c_int32(top_k),
                                    C.c_float(temperature), _ptr(uniforms), _ptr(out), _stream_ptr(stream)))
    return out


# ---------------------------------------------------------------------------------------------
# serving many requests from one paged cache
# ---------------------------------------------------------------------------------------------
# These calls are made every step, so their checks are written for speed: one condition over all tensors, attribute by attribute
# (0.05 us each), and a search for the culprit only where it fails.
_I32, _F32, _F16, _BF16, _I16, _U8 = torch.int32, torch.float32, torch.float16, torch.bfloat16, torch.int16, torch.uint8


def _refuse(what):
    raise TtsGptError(E_ARG, what)


def _refuse_index(d, **tensors):
    """Says which of the tensors is not a contiguous int32 tensor on device number d, if one is."""
    for name, t in tensors.items():
        if t is not None and (t.dtype is not _I32 or t.get_device() != d or not t.is_contiguous()):
            _refuse("%s must be a contiguous int32 tensor on the same device as the others" % name)


def _run(fn, d, stream, *args):
    """Calls a C entry point with device number d current, on `stream` or torch's current one of that device."""
    if d < 0:
        _refuse("tensors must be on a CUDA device")
    st = torch._C._cuda_getCurrentRawStream(d) if stream is None else stream.cuda_stream
    if d == torch._C._cuda_getDevice():
        rc = fn(*args, st)
    else:
        with torch.cuda.device(d):
            rc = fn(*args, st)
    if rc:
        _check(rc)


def _pool(kv_layer, d):
    """(format, pages, heads) of one layer's pool: bf16 [pages, 2, heads, 64, 64], or bytes [pages, 2, heads, 4352]."""
    sh = kv_layer.shape
    if kv_layer.get_device() == d and kv_layer.is_contiguous():
        t = kv_layer.dtype
        if (t is _BF16 or t is _I16) and len(sh) == 5 and sh[1] == 2 and sh[3] == 64 and sh[4] == 64:
            return 0, sh[0], sh[2]
        if t is _U8 and len(sh) == 4 and sh[1] == 2 and sh[3] == 4352:
            return 1, sh[0], sh[2]
    _refuse("kv_layer must be a contiguous bf16 tensor [pages, 2, heads, 64, 64] or uint8 tensor [pages, 2, heads, 4352] on the same device as the others")


def op_page_tables(new_len, ctx_len, page_table, free_pages, free_top, row_start, row_stream, row_pos, row_slot, info,
                   stream_ids=None, shared_pages=None, ctx_len_out=None, free_top_out=None, stream=None):
    """Page lists and slot maps of a pass from the requests' lengths; everything int32 on one device, written in place.  row_stream,
    row_pos and row_slot hold as many rows as the pass may have.  ctx_len_out, free_top_out: None updates ctx_len, free_top.
    info: 8 values, zero at first; info[0] is the status the lengths lead to, which lives on the device like they do."""
    d, n, streams, rows = new_len.get_device(), new_len.numel(), ctx_len.numel(), row_stream.numel()
    if ctx_len_out is None:
        ctx_len_out = ctx_len
    if free_top_out is None:
        free_top_out = free_top
    ids = shared = None
    n_shared = 0
    fine = (new_len.dtype is ctx_len.dtype is page_table.dtype is free_pages.dtype is free_top.dtype is row_start.dtype is row_stream.dtype is row_pos.dtype
            is row_slot.dtype is info.dtype is ctx_len_out.dtype is free_top_out.dtype is _I32
            and ctx_len.get_device() == page_table.get_device() == free_pages.get_device() == free_top.get_device() == row_start.get_device()
            == row_stream.get_device() == row_pos.get_device() == row_slot.get_device() == info.get_device() == ctx_len_out.get_device()
            == free_top_out.get_device() == d
            and new_len.is_contiguous() and ctx_len.is_contiguous() and page_table.is_contiguous() and free_pages.is_contiguous() and row_start.is_contiguous()
            and row_stream.is_contiguous() and row_pos.is_contiguous() and row_slot.is_contiguous() and info.is_contiguous() and ctx_len_out.is_contiguous())
    if stream_ids is not None:
        fine = fine and stream_ids.dtype is _I32 and stream_ids.get_device() == d and stream_ids.is_contiguous() and stream_ids.numel() == n
        ids = stream_ids.data_ptr()
    if shared_pages is not None:
        fine = fine and shared_pages.dtype is _I32 and shared_pages.get_device() == d and shared_pages.is_contiguous()
        shared, n_shared = shared_pages.data_ptr(), shared_pages.numel()
    shape = page_table.shape
    if not (fine and len(shape) == 2 and shape[0] == streams == ctx_len_out.numel() and row_pos.numel() == rows == row_slot.numel() and row_start.numel() > n
            and info.numel() >= 8 and free_top.numel() and free_top_out.numel()):
        _refuse_index(d, new_len=new_len, ctx_len=ctx_len, page_table=page_table, free_pages=free_pages, free_top=free_top, row_start=row_start,
                      row_stream=row_stream, row_pos=row_pos, row_slot=row_slot, info=info, stream_ids=stream_ids, shared_pages=shared_pages,
                      ctx_len_out=ctx_len_out, free_top_out=free_top_out)
        _refuse("page_table must be [streams, pages of a stream], ctx_len [streams], stream_ids as long as new_len, row_start longer, "
                "row_stream, row_pos and row_slot of one length, info 8 long")
    _run((_lib or load()).tts_gpt_op_page_tables, d, stream, n, ids, new_len.data_ptr(), streams, ctx_len.data_ptr(), ctx_len_out.data_ptr(), free_pages.numel(),
         free_pages.data_ptr(), free_top.data_ptr(), free_top_out.data_ptr(), n_shared, shared, shape[1], page_table.data_ptr(), rows, row_start.data_ptr(),
         row_stream.data_ptr(), row_pos.data_ptr(), row_slot.data_ptr(), info.data_ptr())


def op_kv_append(k, v, kv_layer, row_slot, stream=None):
    """K and V rows [R, heads * 64] (fp32 or bf16; rows may be strided) into their slots of the pool."""
    d, t, shape = k.get_device(), k.dtype, k.shape
    fmt, pages, heads = _pool(kv_layer, d)
    if v.dtype is not t or t is _F16 or t not in _TYPES or v.shape != shape or len(shape) != 2 or shape[1] != heads * 64 or v.get_device() != d:
        _refuse("k and v must be [R, %d] of one type, fp32 or bf16, on one device" % (heads * 64))
    (ks, k1), (vs, v1), R = k.stride(), v.stride(), shape[0]
    if k1 != 1 or v1 != 1:
        _refuse("rows of k and v must be contiguous")
    if R == 1:
        ks = vs = heads * 64                   # the stride of a single row addresses nothing
    if row_slot.dtype is not _I32 or row_slot.get_device() != d or not row_slot.is_contiguous() or row_slot.numel() < R:
        _refuse("row_slot must be a contiguous int32 tensor of at least R values on the same device")
    _run((_lib or load()).tts_gpt_op_kv_append, d, stream, R, heads, _TYPES[t], k.data_ptr(), ks, v.data_ptr(), vs, row_slot.data_ptr(), fmt, pages,
         kv_layer.data_ptr())


def _on(stream):
    """Where memory that a call makes for itself belongs: the stream that the call runs on."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _scratch(scratch, d):
    if scratch.dtype is not _U8 or scratch.get_device() != d or not scratch.is_contiguous():
        _refuse("scratch must be a contiguous uint8 tensor on the same device")
    return scratch.data_ptr(), scratch.numel()


def debug_expire_op(cta, limit_us=1000):
    """Test aid: copies of CTA `cta` never count as complete in this thread's next attention calls; -1: as usual again."""
    _check(load().tts_gpt_debug_expire_op(C.c_int32(cta), C.c_uint32(limit_us)))


def op_attention_shared_scratch(R, n_head, n_kv_head, device):
    n = C.c_size_t(0)
    _check(load().tts_gpt_op_attention_shared_scratch_bytes(C.c_int32(R), C.c_int32(n_head), C.c_int32(n_kv_head), C.byref(n)))
    return torch.zeros(n.value, dtype=torch.uint8, device=device)


def op_attention_shared(q, kv_layer, page_table, row_stream, row_pos, n_shared, scratch=None, out=None, stream=None):
    """Attention of rows q [R, heads * 64] (fp32 or bf16) over a paged cache whose page lists all begin with the same n_shared
    pages.  The pool may have fewer heads than q.  Returns bf16 bits [R, heads * 64], or `out`.  Rows that are not computed since a
    wait inside a kernel ran out are NaN (others may be); the first int32 of `scratch` is then 1, and it must be zeroed before its next use."""
    d, t, shape = q.get_device(), q.dtype, q.shape
    fmt, pages, kv_heads = _pool(kv_layer, d)
    if len(shape) != 2 or shape[1] % 64 or t is _F16 or t not in _TYPES:
        _refuse("q must be [R, heads * 64], fp32 or bf16")
    (qs, q1), R, heads = q.stride(), shape[0], shape[1] // 64
    if q1 != 1:
        _refuse("rows of q must be contiguous")
    if R == 1:
        qs = heads * 64                        # the stride of a single row addresses nothing
    lists = page_table.shape
    if not (page_table.dtype is row_stream.dtype is row_pos.dtype is _I32 and page_table.get_device() == row_stream.get_device() == row_pos.get_device() == d
            and page_table.is_contiguous() and row_stream.is_contiguous() and row_pos.is_contiguous() and len(lists) == 2 and row_stream.numel() >= R
            and row_pos.numel() >= R):
        _refuse_index(d, page_table=page_table, row_stream=row_stream, row_pos=row_pos)
        _refuse("page_table must be [streams, pages of a stream], row_stream and row_pos at least R long")
    if out is None:
        with _on(stream):
            out = torch.empty(shape, dtype=_I16, device=q.device)
    elif out.shape != shape or (out.dtype is not _BF16 and out.dtype is not _I16) or out.get_device() != d or not out.is_contiguous():
        _refuse("out must be a contiguous bf16 tensor of q's shape on the same device")
    if scratch is None:
        with _on(stream):
            scratch = op_attention_shared_scratch(R, heads, kv_heads, q.device)
    sp, sn = _scratch(scratch, d)
    _run((_lib or load()).tts_gpt_op_attention_shared, d, stream, R, heads, kv_heads, _TYPES[t], q.data_ptr(), qs, fmt, pages, kv_layer.data_ptr(), n_shared,
         page_table.data_ptr(), lists[1], row_stream.data_ptr(), row_pos.data_ptr(), out.data_ptr(), sp, sn)
    return out


def op_attention_cross_scratch(device):
    n = C.c_size_t(0)
    _check(load().tts_gpt_op_attention_cross_scratch_bytes(C.byref(n)))
    return torch.zeros(n.value, dtype=torch.uint8, device=device)


def op_attention_cross(q, k, v, q_start, k_start, q_max, scale=0.125, scratch=None, out=None, stream=None):
    """Attention of ragged sequences of queries q [rows, heads, 64] to keys and values k, v [rows, kv heads, 64] of other lengths, bf16
    or fp16; sequence i has rows q_start[i] .. q_start[i+1]-1 of q and k_start[i] .. k_start[i+1]-1 of k and v, whose rows and heads
    may be strided.  q_max: at least the longest sequence of queries.  Returns [rows, heads, 64] (rows of no sequence undefined), or `out`
    (in which they are left as they were).  NaN rows and scratch as for op_attention_shared."""
    d, t, shape, kshape = q.get_device(), q.dtype, q.shape, k.shape
    if (t is not _BF16 and t is not _F16) or not (k.dtype is v.dtype is t) or len(shape) != 3 or len(kshape) != 3 or v.shape != kshape or shape[2] != 64 \
            or kshape[2] != 64 or k.get_device() != d or v.get_device() != d:
        _refuse("q must be [rows, heads, 64], k and v [rows, kv heads, 64], all bf16 or all fp16, on one device")
    (qs, qh, q1), (kr, kh, k1), (vr, vh, v1) = q.stride(), k.stride(), v.stride()
    rows, heads, _ = shape
    k_rows, kv_heads, _ = kshape
    if q1 != 1 or k1 != 1 or v1 != 1 or (heads > 1 and qh != 64):
        _refuse("heads of q, and the 64 values of a head of k and v, must be contiguous")
    # strides of a single row or head address nothing
    if rows == 1:
        qs = heads * 64
    if k_rows <= 1:
        kr = vr = 64
    if kv_heads == 1:
        kh = vh = 64
    n = q_start.numel() - 1
    if not (q_start.dtype is k_start.dtype is _I32 and q_start.get_device() == k_start.get_device() == d and q_start.is_contiguous() and k_start.is_contiguous()
            and n >= 1 and k_start.numel() == n + 1):
        _refuse_index(d, q_start=q_start, k_start=k_start)
        _refuse("q_start and k_start must have one value more than there are sequences")
    if out is None:
        with _on(stream):
            out = torch.empty(shape, dtype=t, device=q.device)
    elif out.shape != shape or out.dtype is not t or out.get_device() != d or not out.is_contiguous():
        _refuse("out must be a contiguous tensor of q's shape and type on the same device")
    if scratch is None:
        with _on(stream):
            scratch = op_attention_cross_scratch(q.device)
    sp, sn = _scratch(scratch, d)
    _run((_lib or load()).tts_gpt_op_attention_cross, d, stream, n, heads, kv_heads, _TYPES[t], rows, q.data_ptr(), qs, k_rows, k.data_ptr(), kr, kh,
         v.data_ptr(), vr, vh, q_start.data_ptr(), k_start.data_ptr(), q_max, scale, out.data_ptr(), sp, sn)
    return out


# ---------------------------------------------------------------------------------------------
# several drafted tokens a step
# ---------------------------------------------------------------------------------------------
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}


def op_rope_frequencies(n_rot, base=10000.0, scaling="none", factor=1.0, original=0, low=1.0, high=None, inv_freq=None, device="cuda"):
    """The table op_rope_kv_append takes for heads whose first n_rot values are rotated, and what cosine and sine are multiplied by.  Pair i turns by
    base ** (-2 i / n_rot) radians a position, stretched by ``scaling``: "none", "linear", "ntk", "yarn" (high: 32 turns) or "bands" (high: 4); or by
    inv_freq[i] where that is given (a sequence of n_rot / 2 numbers).  Returns (int64 tensor [n_rot / 2] on `device`, float)."""
    if not isinstance(n_rot, int) or n_rot < 2 or n_rot > 64 or n_rot % 2:
        _refuse("n_rot must be even, 2 to 64")
    given = None
    if inv_freq is not None:
        kind, values = 5, [float(w) for w in inv_freq]
        if len(values) != n_rot // 2:
            _refuse("inv_freq must have n_rot / 2 values")
        given = (C.c_double * len(values))(*values)
    elif scaling in ROPE_SCALINGS:
        kind = ROPE_SCALINGS[scaling]
    else:
        _refuse("scaling must be one of %s" % ", ".join(ROPE_SCALINGS))
    turns, magnitude = (C.c_uint64 * (n_rot // 2))(), C.c_float(1.0)
    _check((_lib or load()).tts_gpt_op_rope_frequencies(n_rot, kind, base, factor, original, low, (32.0 if scaling == "yarn" else 4.0) if high is None else high, given, turns,
                                                        C.byref(magnitude)))
    table = torch.from_numpy(np.frombuffer(turns, dtype=np.int64).copy())
    return table.to(device), magnitude.value


def op_rope_kv_append(q, k, v, kv_layer, row_slot, row_pos, turns, magnitude=1.0, interleaved=False, q_out=None, stream=None):
    """A pass's rows rotated by their positions row_pos [R]: q [R, heads * 64] to q_out (None: a new bf16 tensor; q itself is fine), K (rotated) and V [R, heads of
    the pool * 64] into their slots.  All fp32 or all bf16, rows may be strided; q_out fp32 or bf16.  turns, magnitude: op_rope_frequencies.  Pairs are
    (i, i + n_rot / 2), or (2i, 2i + 1) where interleaved.  q None: K and V only.  A row without a slot is left out, its q_out included."""
    d, t, shape = k.get_device(), k.dtype, k.shape
    fmt, pages, heads = _pool(kv_layer, d)
    if (t is not _F32 and t is not _BF16 and t is not _I16) or v.dtype is not t or len(shape) != 2 or shape[1] != heads * 64 or v.shape != shape or v.get_device() != d:
        _refuse("k and v must be [R, %d] of one type, fp32 or bf16, on one device" % (heads * 64))
    (ks, k1), (vs, v1), R = k.stride(), v.stride(), shape[0]
    if k1 != 1 or v1 != 1:
        _refuse("rows of k and v must be contiguous")
    if R == 1:
        ks = vs = heads * 64                   # the stride of a single row addresses nothing
    if not (row_slot.dtype is row_pos.dtype is _I32 and row_slot.get_device() == row_pos.get_device() == d and row_slot.is_contiguous() and row_pos.is_contiguous()
            and row_slot.numel() >= R and row_pos.numel() >= R):
        _refuse("row_slot and row_pos must be contiguous int32 tensors of at least R values on the same device")
    if turns.dtype is not torch.int64 or turns.get_device() != d or not turns.is_contiguous():
        _refuse("turns must be a contiguous int64 tensor on the same device")
    qp = op = None
    qh = qs = os_ = 0
    ot = _BF16
    if q is not None:
        qshape = q.shape
        if q.dtype is not t or len(qshape) != 2 or qshape[0] != R or qshape[1] % 64 or not qshape[1] or q.get_device() != d:
            _refuse("q must be [R, heads * 64] of the type of k and v on the same device")
        if q_out is None:
            with _on(stream):
                q_out = torch.empty(qshape, dtype=_BF16, device=q.device)
        ot = q_out.dtype
        if (ot is not _F32 and ot is not _BF16 and ot is not _I16) or q_out.shape != qshape or q_out.get_device() != d:
            _refuse("q_out must be of q's shape, fp32 or bf16, on the same device")
        (qs, q1), (os_, o1), qh = q.stride(), q_out.stride(), qshape[1] // 64
        if q1 != 1 or o1 != 1:
            _refuse("rows of q and q_out must be contiguous")
        if R == 1:
            qs = os_ = qh * 64
        qp, op = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        _refuse("there is no q for q_out")
    _run((_lib or load()).tts_gpt_op_rope_kv_append, d, stream, R, qh, heads, _TYPES[t], qp, qs, k.data_ptr(), ks, v.data_ptr(), vs, row_pos.data_ptr(), row_slot.data_ptr(),
         2 * turns.numel(), turns.data_ptr(), 1 if interleaved else 0, magnitude, _TYPES[ot], op, os_, fmt, pages, kv_layer.data_ptr())
    return q_out


def _trees(d, row_start, stream_ids, kv_len):
    """Number of trees of a call, and the address of their streams' numbers."""
    n = row_start.numel() - 1
    if not (row_start.dtype is kv_len.dtype is _I32 and row_start.get_device() == kv_len.get_device() == d and row_start.is_contiguous() and kv_len.is_contiguous() and n >= 1):
        _refuse_index(d, row_start=row_start, kv_len=kv_len)
        _refuse("row_start must have one value more than there are trees")
    if stream_ids is None:
        return n, None
    if stream_ids.dtype is not _I32 or stream_ids.get_device() != d or not stream_ids.is_contiguous() or stream_ids.numel() != n:
        _refuse("stream_ids must be a contiguous int32 tensor with a value for each tree on the same device")
    return n, stream_ids.data_ptr()


def op_tree_tables(parent, row_start, kv_len, tree_mask, row_pos, info, stream_ids=None, stream=None):
    """Masks [R, words] and positions [R] of trees from the parents [R] (numbers inside the tree, -1: none); everything int32 on one device, written in
    place.  info[0], zero at first, becomes the lowest code of a tree with something wrong, which is left as it was."""
    d, R = parent.get_device(), parent.numel()
    n, ids = _trees(d, row_start, stream_ids, kv_len)
    shape = tree_mask.shape
    if not (parent.dtype is tree_mask.dtype is row_pos.dtype is info.dtype is _I32 and tree_mask.get_device() == row_pos.get_device() == info.get_device() == d
            and parent.is_contiguous() and tree_mask.is_contiguous() and row_pos.is_contiguous() and info.is_contiguous() and len(shape) == 2 and shape[0] == R
            and row_pos.numel() == R and info.numel() >= 1):
        _refuse_index(d, parent=parent, tree_mask=tree_mask, row_pos=row_pos, info=info)
        _refuse("parent and row_pos must have a value, and tree_mask a row, for each row")
    _run((_lib or load()).tts_gpt_op_tree_tables, d, stream, n, R, row_start.data_ptr(), ids, kv_len.numel(), kv_len.data_ptr(), parent.data_ptr(), shape[1], tree_mask.data_ptr(),
         row_pos.data_ptr(), info.data_ptr())


def op_attention_tree_scratch(device):
    n = C.c_size_t(0)
    _check(load().tts_gpt_op_attention_tree_scratch_bytes(C.byref(n)))
    return torch.zeros(n.value, dtype=torch.uint8, device=device)


def op_attention_tree(q, kv_layer, page_table, row_start, kv_len, tree_mask, t_max, stream_ids=None, scale=0.125, scratch=None, out=None, stream=None):
    """Attention of trees of drafted tokens: rows q [R, heads * 64] (fp32 or bf16), of which tree i has row_start[i] .. row_start[i + 1] - 1, to the committed keys of
    their streams and to the nodes of the tree that their masks [R, words] name.  kv_len counts a stream's tokens with the tree's nodes; t_max: at least the
    largest tree.  Returns bf16 [R, heads * 64] (rows of no tree undefined), or `out` (in which they are left as they were).  NaN rows and scratch as for
    op_attention_shared."""
    d, t, shape = q.get_device(), q.dtype, q.shape
    fmt, pages, kv_heads = _pool(kv_layer, d)
    if len(shape) != 2 or shape[1] % 64 or (t is not _F32 and t is not _BF16 and t is not _I16):
        _refuse("q must be [R, heads * 64], fp32 or bf16")
    (qs, q1), R, heads = q.stride(), shape[0], shape[1] // 64
    if q1 != 1:
        _refuse("rows of q must be contiguous")
    if R == 1:
        qs = heads * 64                        # the stride of a single row addresses nothing
    n, ids = _trees(d, row_start, stream_ids, kv_len)
    lists, words = page_table.shape, tree_mask.shape
    if not (page_table.dtype is tree_mask.dtype is _I32 and page_table.get_device() == tree_mask.get_device() == d and page_table.is_contiguous() and tree_mask.is_contiguous()
            and len(lists) == 2 and lists[0] == kv_len.numel() and len(words) == 2 and words[0] >= R):
        _refuse_index(d, page_table=page_table, tree_mask=tree_mask)
        _refuse("page_table must be [streams, pages of a stream] for the streams of kv_len, tree_mask [R, words]")
    if out is None:
        with _on(stream):
            out = torch.empty(shape, dtype=_BF16, device=q.device)
    elif out.shape != shape or (out.dtype is not _BF16 and out.dtype is not _I16) or out.get_device() != d or not out.is_contiguous():
        _refuse("out must be a contiguous bf16 tensor of q's shape on the same device")
    if scratch is None:
        with _on(stream):
            scratch = op_attention_tree_scratch(q.device)
    sp, sn = _scratch(scratch, d)
    _run((_lib or load()).tts_gpt_op_attention_tree, d, stream, n, R, heads, kv_heads, _TYPES[t], q.data_ptr(), qs, fmt, pages, kv_layer.data_ptr(), lists[0], page_table.data_ptr(),
         lists[1], row_start.data_ptr(), ids, kv_len.data_ptr(), words[1], tree_mask.data_ptr(), t_max, scale, out.data_ptr(), sp, sn)
    return out


def op_tree_accept(draft, target, parent, row_start, kv_len, page_table, free_pages, free_top, path, n_accepted, next_token, info, stream_ids=None, kv_len_out=None,
                   free_top_out=None, stream=None):
    """The path from node 0 through children whose drafted token is the model's (target, by row) after their parent; everything int32 on one device, written in
    place: path [R] (rows of accepted nodes at the head of the tree's rows, then -1), n_accepted and next_token by tree, the streams' lengths without the other nodes
    (kv_len_out, None: kv_len), and unused pages back onto the stack (free_pages, free_top_out, None: free_top).  info: 8 values, zero at first; info[0] is the status:
    where it is not 0, path is -1 in all trees' rows and lengths and stack are as they were."""
    d, R = draft.get_device(), draft.numel()
    n, ids = _trees(d, row_start, stream_ids, kv_len)
    if kv_len_out is None:
        kv_len_out = kv_len
    if free_top_out is None:
        free_top_out = free_top
    lists = page_table.shape
    if not (draft.dtype is target.dtype is parent.dtype is page_table.dtype is free_pages.dtype is free_top.dtype is path.dtype is n_accepted.dtype is next_token.dtype is info.dtype
            is kv_len_out.dtype is free_top_out.dtype is _I32
            and target.get_device() == parent.get_device() == page_table.get_device() == free_pages.get_device() == free_top.get_device() == path.get_device()
            == n_accepted.get_device() == next_token.get_device() == info.get_device() == kv_len_out.get_device() == free_top_out.get_device() == d
            and draft.is_contiguous() and target.is_contiguous() and parent.is_contiguous() and page_table.is_contiguous() and free_pages.is_contiguous() and path.is_contiguous()
            and n_accepted.is_contiguous() and next_token.is_contiguous() and info.is_contiguous() and kv_len_out.is_contiguous()
            and target.numel() == parent.numel() == path.numel() == R and len(lists) == 2 and lists[0] == kv_len.numel() == kv_len_out.numel()
            and n_accepted.numel() >= n and next_token.numel() >= n and info.numel() >= 8 and free_top.numel() and free_top_out.numel()):
        _refuse_index(d, draft=draft, target=target, parent=parent, page_table=page_table, free_pages=free_pages, free_top=free_top, path=path, n_accepted=n_accepted,
                      next_token=next_token, info=info, kv_len_out=kv_len_out, free_top_out=free_top_out)
        _refuse("draft, target, parent and path must be of one length, page_table [streams, pages of a stream] for the streams of kv_len and kv_len_out, n_accepted and "
                "next_token as long as there are trees, info 8 long")
    _run((_lib or load()).tts_gpt_op_tree_accept, d, stream, n, R, row_start.data_ptr(), ids, draft.data_ptr(), target.data_ptr(), parent.data_ptr(), lists[0], kv_len.data_ptr(),
         kv_len_out.data_ptr(), page_table.data_ptr(), lists[1], free_pages.numel(), free_pages.data_ptr(), free_top.data_ptr(), free_top_out.data_ptr(), path.data_ptr(),
         n_accepted.data_ptr(), next_token.data_ptr(), info.data_ptr())


def op_kv_move(kv_layers, row_start, path, row_slot, stream=None):
    """K and V of accepted nodes to the slots of their tree's first rows, in one layer's pool or in several [layers, ...] (which may be strided)."""
    d, shape, u8 = kv_layers.get_device(), kv_layers.shape, kv_layers.dtype is _U8
    if len(shape) == (5 if u8 else 6):
        layers, pages, heads = shape[0], shape[1], shape[3]
        strides = kv_layers.stride()
        # of a layer that is contiguous and has a format's shape
        sound = ((shape[2:] == (2, heads, 4352) and strides[1:] == (8704 * heads, 4352 * heads, 4352, 1)) if u8 else
                 (shape[2:] == (2, heads, 64, 64) and strides[1:] == (8192 * heads, 4096 * heads, 4096, 64, 1) and kv_layers.dtype in (_BF16, _I16)))
        if sound and layers:
            fmt, stride = (1, strides[0]) if u8 else (0, 2 * strides[0])
        else:                                  # (a size of one may have any stride)
            if not layers:
                _refuse("there must be a layer")
            fmt, pages, heads = _pool(kv_layers[0], d)
            stride = strides[0] * kv_layers.element_size()
    else:
        layers, stride = 1, 0
        fmt, pages, heads = _pool(kv_layers, d)
    n, R = row_start.numel() - 1, path.numel()
    if not (row_start.dtype is path.dtype is row_slot.dtype is _I32 and row_start.get_device() == path.get_device() == row_slot.get_device() == d and row_start.is_contiguous()
            and path.is_contiguous() and row_slot.is_contiguous() and n >= 1 and row_slot.numel() >= R):
        _refuse_index(d, row_start=row_start, path=path, row_slot=row_slot)
        _refuse("row_start must have one value more than there are trees, row_slot one for each of path's")
    _run((_lib or load()).tts_gpt_op_kv_move, d, stream, n, R, row_start.data_ptr(), path.data_ptr(), row_slot.data_ptr(), heads, fmt, pages, layers, stride, kv_layers.data_ptr())


def bf16_bits_tensor_to_f32(t: torch.Tensor) -> torch.Tensor:
    """int16 tensor of bf16 bit patterns -> float32 tensor (host or device)."""
    return t.view(torch.bfloat16).to(torch.float32)
