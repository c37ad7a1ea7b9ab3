"""ctypes binding of ``libaio.so`` (C ABI in ``include/aio.h``).

Argument marshalling only: every step of the decode path runs in the HIP
kernels of ``libaio.so``.  Torch provides device memory and streams.  If the
library is missing this module raises instead of computing anything else.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libaio.so")

AIO_OK, AIO_EINVAL, AIO_ERANGE, AIO_EUNSUPPORTED, AIO_EHIP, AIO_ENOMEM, AIO_EDEVICE = \
    0, -1, -2, -3, -4, -5, -6
AIO_WFMT_BF16, AIO_WFMT_INT8 = 0, 1
AIO_MAX_VERIFY_ROWS = 10
AIO_F32, AIO_BF16 = 0, 1
AIO_MAX_TOP = 32
LINEARS = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")
SCALES = ("sq", "sk", "sv", "so", "s_gate", "s_up", "s_down")


class aio_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads",
                                              "head_dim", "ffn_dim", "vocab", "max_ctx",
                                              "max_verify", "wfmt")] + \
               [("rms_eps", ctypes.c_float), ("rope_base", ctypes.c_float)]


class aio_layer_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("attn_norm", "ffn_norm") + LINEARS + SCALES]


class aio_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("lm_head", ctypes.c_void_p), ("s_lm_head", ctypes.c_void_p),
                ("layers", ctypes.POINTER(aio_layer_weights))]


class aio_pld_stats(ctypes.Structure):
    _fields_ = [("forwards", ctypes.c_int32), ("verifies", ctypes.c_int32),
                ("drafted", ctypes.c_int32), ("accepted", ctypes.c_int32)]


class aio_spec_stats(ctypes.Structure):
    _fields_ = [("rounds", ctypes.c_int32), ("drafted", ctypes.c_int32),
                ("accepted", ctypes.c_int32), ("draft_steps", ctypes.c_int32)]


class aio_paged_kv(ctypes.Structure):
    _fields_ = [("k_dev", ctypes.c_void_p), ("v_dev", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim")]


class aio_paged_pool(ctypes.Structure):
    _fields_ = [("first", aio_paged_kv), ("layer_stride", ctypes.c_int64),
                ("n_layers", ctypes.c_int32)]


class aio_packed_kv(ctypes.Structure):
    _fields_ = [("k_dev", ctypes.c_void_p), ("v_dev", ctypes.c_void_p),
                ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("n_rows", "n_kv_heads", "head_dim")]


class aio_seqs(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("cu_q_dev", ctypes.c_void_p),
                ("lens_dev", ctypes.c_void_p), ("table_dev", ctypes.c_void_p),
                ("table_stride", ctypes.c_int32), ("cu_k_dev", ctypes.c_void_p)]


class aio_q8_kv(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_dev", "v_dev", "k_exp_dev", "v_exp_dev")] + \
               [(n, ctypes.c_int64) for n in ("page_stride", "head_stride", "exp_page_stride",
                                              "exp_head_stride")] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim")]


class aio_prefixes(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("max_prefix", ctypes.c_int32),
                ("cu_seqs_dev", ctypes.c_void_p), ("prefix_lens_dev", ctypes.c_void_p)]


class aio_qk_rows(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q_dev", "k_dev", "q_out_dev", "k_out_dev")] + \
               [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "q_out_stride",
                                              "k_out_stride")] + \
               [(n, ctypes.c_int32) for n in ("dtype", "n_rows", "n_heads", "n_kv_heads",
                                              "head_dim")]


class aio_attn(ctypes.Structure):
    _fields_ = [("q_dev", ctypes.c_void_p), ("out_dev", ctypes.c_void_p),
                ("lse_dev", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("scale", ctypes.c_float)]


class AioError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__("%s failed: %d (%s)%s" % (
            what, code, aio_strerror(code),
            "" if code != AIO_EHIP else ", hipError %d" % aio_last_hip_error()))


_lib = None


def lib():
    """The loaded library; raises if it was not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libaio.so is not built (run python -m paper_2604_09752_amd.build)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        P = ctypes.POINTER
        L.aio_kv_bytes.argtypes = [P(aio_config)]
        L.aio_kv_bytes.restype = ctypes.c_size_t
        L.aio_workspace_bytes.argtypes = [P(aio_config)]
        L.aio_workspace_bytes.restype = ctypes.c_size_t
        L.aio_check_config.argtypes = [P(aio_config)]
        L.aio_check_decode.argtypes = [P(aio_config), i32, i32]
        L.aio_check_verify.argtypes = [P(aio_config), i32, vp, i32, i32]
        L.aio_strerror.argtypes = [ctypes.c_int]
        L.aio_strerror.restype = ctypes.c_char_p
        L.aio_last_hip_error.restype = ctypes.c_int
        L.aio_model_load.argtypes = [P(aio_config), P(aio_weights), vp, vp, vp, P(vp)]
        L.aio_model_free.argtypes = [vp]
        L.aio_model_free.restype = None
        L.aio_decode_step.argtypes = [vp, i32, i32, vp]
        L.aio_verify.argtypes = [vp, i32, vp, i32, i32, vp]
        L.aio_argmax.argtypes = [vp, vp, i32, i32, vp]
        L.aio_decode_greedy.argtypes = [vp, i32, i32, i32, vp, vp]
        L.aio_profile_step.argtypes = [vp, i32, i32, vp, vp, i32, P(i32)]
        L.aio_trace_step.argtypes = [vp, i32, i32, vp, vp, i32, P(i32)]
        L.aio_device_status.argtypes = [vp, P(i32)]
        L.aio_trace_barriers.argtypes = [vp, i32, i32, vp, vp, vp, i32, P(i32), P(i32)]
        L.aio_uses_step_kernel.argtypes = [vp]
        L.aio_pld_match.argtypes = [vp, i32, i32, i32, i32, vp, P(i32)]
        L.aio_pld_generate.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp,
                                       P(aio_pld_stats)]
        L.aio_tune_step.argtypes = [vp, i32, i32, vp, i32]
        L.aio_prefill.argtypes = [vp, vp, i32, i32, vp]
        L.aio_prefill_noalloc.argtypes = [vp, vp, i32, i32, vp]
        L.aio_prefill_noalloc_rows.argtypes = [P(aio_config)]
        L.aio_category_entropy.argtypes = [vp, vp, vp, i32, vp]
        L.aio_category_entropy.restype = i32
        L.aio_probe_route.argtypes = [vp, i32, i32, i32, i32, ctypes.c_float,
                                      P(ctypes.c_float), P(i32)]
        L.aio_spec_generate.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                        P(aio_spec_stats)]
        i64, sz = ctypes.c_int64, ctypes.c_size_t
        L.aio_attn_workspace_bytes.argtypes = [vp, i32, i32, i32]
        L.aio_attn_workspace_bytes.restype = sz
        # (structs by address: byref of one, or its bytes)
        L.aio_paged_attention.argtypes = [vp, vp, vp, vp, sz, vp]
        L.aio_packed_attention.argtypes = [vp, vp, vp, vp, sz, vp]
        L.aio_page_append.argtypes = [vp, vp, vp, vp, i32, i64, i64, vp]
        L.aio_q8_append.argtypes = [vp, vp, vp, vp, i32, i64, i64, vp]
        L.aio_q8_attention.argtypes = [vp, vp, vp, vp, sz, vp]
        L.aio_prefix_attention.argtypes = [vp, vp, vp, vp, vp, sz, vp]
        L.aio_q8_prefix_attention.argtypes = [vp, vp, vp, vp, vp, sz, vp]
        L.aio_q8_workspace_bytes.argtypes = [vp, i32, i32, i32]
        L.aio_q8_workspace_bytes.restype = sz
        L.aio_prefix_workspace_bytes.argtypes = [vp, vp, i32, i32, i32]
        L.aio_prefix_workspace_bytes.restype = sz
        L.aio_qk_norm_rope.argtypes = [vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp]
        L.aio_page_copy.argtypes = [vp, i32, i64, i32, i64, i64, vp, vp, i32, vp]
        L.aio_logprobs.argtypes = [vp, i32, i32, i32, i64, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.aio_logprobs_workspace_bytes.argtypes = [i32, i32, i32]
        L.aio_logprobs_workspace_bytes.restype = sz
        L.aio_paged_forward.argtypes = [vp, P(aio_paged_pool), i32, vp, vp, vp, i32, vp, vp, i32,
                                        vp, vp, sz]
        L.aio_paged_forward_bytes.argtypes = [P(aio_config), i32, i32, i32]
        L.aio_paged_forward_bytes.restype = sz
        L.aio_pages_create.argtypes = [i32, i32, i32, P(vp)]
        L.aio_pages_destroy.argtypes = [vp]
        L.aio_pages_destroy.restype = None
        L.aio_pages_open.argtypes = [vp, P(i32)]
        L.aio_pages_close.argtypes = [vp, i32]
        L.aio_pages_fork.argtypes = [vp, i32, P(i32)]
        L.aio_pages_extend.argtypes = [vp, i32, i32, P(i32), P(i32), P(i32)]
        L.aio_pages_truncate.argtypes = [vp, i32, i32]
        L.aio_pages_compact.argtypes = [vp, vp, vp, i32, P(i32)]
        L.aio_pages_row.argtypes = [vp, i32, vp, i32, P(i32)]
        L.aio_pages_free.argtypes = [vp]
        _lib = L
    return _lib


def make_config(cfg) -> aio_config:
    """aio_config from any object with the usual shape attributes."""
    c = aio_config()
    for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "ffn_dim", "vocab",
              "max_ctx", "max_verify"):
        setattr(c, n, int(getattr(cfg, n)))
    if c.max_verify > AIO_MAX_VERIFY_ROWS:
        c.max_verify = AIO_MAX_VERIFY_ROWS
    c.wfmt = AIO_WFMT_INT8 if getattr(cfg, "wfmt", "bf16") == "int8" else AIO_WFMT_BF16
    c.rms_eps = float(cfg.rms_eps)
    c.rope_base = float(cfg.rope_base)
    return c


def _ptr(t) -> int | None:
    if t is None:
        return None
    return t.data_ptr()


def _check(rc: int, what: str):
    if rc != AIO_OK:
        raise AioError(rc, what)


# ------------------------------------------------------------- pure host calls

def aio_kv_bytes(c: aio_config) -> int:
    return int(lib().aio_kv_bytes(ctypes.byref(c)))


def aio_workspace_bytes(c: aio_config) -> int:
    return int(lib().aio_workspace_bytes(ctypes.byref(c)))


def aio_check_config(c: aio_config) -> int:
    return int(lib().aio_check_config(ctypes.byref(c) if c is not None else None))


def aio_check_decode(c: aio_config, token: int, pos: int) -> int:
    return int(lib().aio_check_decode(ctypes.byref(c), token, pos))


def aio_check_verify(c: aio_config, token: int, drafts, k: int, pos: int) -> int:
    arr = None if drafts is None else np.ascontiguousarray(drafts, dtype=np.int32)
    return int(lib().aio_check_verify(ctypes.byref(c), token,
                                      None if arr is None else arr.ctypes.data, k, pos))


def aio_strerror(code: int) -> str:
    return lib().aio_strerror(code).decode()


def aio_last_hip_error() -> int:
    return int(lib().aio_last_hip_error())


# ------------------------------------------------------------ model handles

def aio_model_load(c: aio_config, w: aio_weights, kv: torch.Tensor, ws: torch.Tensor,
                   stream: int | None) -> int:
    h = ctypes.c_void_p()
    _check(lib().aio_model_load(ctypes.byref(c), ctypes.byref(w), _ptr(kv), _ptr(ws), stream,
                                ctypes.byref(h)), "aio_model_load")
    return h.value


def aio_model_free(handle: int) -> None:
    lib().aio_model_free(handle)


def aio_decode_step(handle: int, token: int, pos: int, logits: torch.Tensor) -> None:
    _check(lib().aio_decode_step(handle, int(token), int(pos), _ptr(logits)), "aio_decode_step")


def aio_verify(handle: int, token: int, drafts, k: int, pos: int, logits: torch.Tensor) -> None:
    arr = np.ascontiguousarray(drafts if drafts is not None else [], dtype=np.int32)
    _check(lib().aio_verify(handle, int(token), arr.ctypes.data if arr.size else None, int(k),
                            int(pos), _ptr(logits)), "aio_verify")


def aio_argmax(handle: int, logits: torch.Tensor, rows: int, n: int, out: torch.Tensor) -> None:
    _check(lib().aio_argmax(handle, _ptr(logits), int(rows), int(n), _ptr(out)), "aio_argmax")


def aio_decode_greedy(handle: int, token: int, pos: int, n_steps: int, tokens: torch.Tensor,
                      logits: torch.Tensor) -> None:
    _check(lib().aio_decode_greedy(handle, int(token), int(pos), int(n_steps), _ptr(tokens),
                                   _ptr(logits)), "aio_decode_greedy")


KERNELS_PER_LAYER = ("qkv", "attn", "merge", "o", "gateup", "down")


def aio_profile_step(handle: int, token: int, pos: int, logits: torch.Tensor,
                     max_kernels: int) -> np.ndarray:
    """Per-kernel event-to-event milliseconds of one decode step."""
    ms = np.zeros(max_kernels, dtype=np.float32)
    n = ctypes.c_int32(0)
    _check(lib().aio_profile_step(handle, int(token), int(pos), _ptr(logits), ms.ctypes.data,
                                  int(max_kernels), ctypes.byref(n)), "aio_profile_step")
    return ms[: n.value].copy()


def aio_trace_step(handle: int, token: int, pos: int, logits: torch.Tensor,
                   max_phases: int) -> np.ndarray:
    """Per-phase microseconds of one step of the persistent kernel."""
    us = np.zeros(max_phases, dtype=np.float64)
    n = ctypes.c_int32(0)
    _check(lib().aio_trace_step(handle, int(token), int(pos), _ptr(logits), us.ctypes.data,
                                int(max_phases), ctypes.byref(n)), "aio_trace_step")
    return us[: n.value].copy()


def aio_trace_barriers(handle: int, token: int, pos: int, logits: torch.Tensor, n_layers: int,
                       max_blocks: int = 1024):
    """(arrive, leave) device-clock times [barrier][workgroup] of one step."""
    cap = (5 * n_layers + 1) * max_blocks
    arr = np.zeros(cap, dtype=np.uint64)
    lev = np.zeros(cap, dtype=np.uint64)
    nb, nk = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().aio_trace_barriers(handle, int(token), int(pos), _ptr(logits), arr.ctypes.data,
                                    lev.ctypes.data, cap, ctypes.byref(nb), ctypes.byref(nk)),
           "aio_trace_barriers")
    n = nb.value * nk.value
    return arr[:n].reshape(nb.value, nk.value), lev[:n].reshape(nb.value, nk.value)


def aio_pld_match(hist, ngram_max: int, ngram_min: int, k: int) -> np.ndarray:
    """Prompt-lookup drafts for the history ``hist`` (pure host call)."""
    h = np.ascontiguousarray(hist, dtype=np.int32)
    out = np.zeros(max(int(k), 1), dtype=np.int32)
    n = ctypes.c_int32(0)
    _check(lib().aio_pld_match(h.ctypes.data if h.size else None, int(h.size), int(ngram_max),
                               int(ngram_min), int(k), out.ctypes.data, ctypes.byref(n)),
           "aio_pld_match")
    return out[: n.value].copy()


def aio_pld_generate(handle: int, history, pos: int, token: int, n_new: int, ngram_max: int,
                     ngram_min: int, k: int, logits: torch.Tensor, argmax_out: torch.Tensor):
    """Greedy generation with prompt-lookup decoding; returns (tokens, stats)."""
    h = np.ascontiguousarray(history, dtype=np.int32)
    assert h.size == pos
    out = np.zeros(int(n_new), dtype=np.int32)
    st = aio_pld_stats()
    _check(lib().aio_pld_generate(handle, h.ctypes.data if h.size else None, int(pos), int(token),
                                  int(n_new), int(ngram_max), int(ngram_min), int(k),
                                  _ptr(logits), _ptr(argmax_out), out.ctypes.data,
                                  ctypes.byref(st)), "aio_pld_generate")
    return out, {f: int(getattr(st, f)) for f, _ in aio_pld_stats._fields_}


def aio_spec_generate(target: int, draft: int, pos: int, token: int, n_new: int, k: int,
                      target_logits: torch.Tensor, draft_logits: torch.Tensor,
                      argmax_out: torch.Tensor, draft_tokens: torch.Tensor):
    """Greedy generation of the target with drafts from the draft model;
    returns (tokens, stats)."""
    out = np.zeros(int(n_new), dtype=np.int32)
    st = aio_spec_stats()
    _check(lib().aio_spec_generate(target, draft, int(pos), int(token), int(n_new), int(k),
                                   _ptr(target_logits), _ptr(draft_logits), _ptr(argmax_out),
                                   _ptr(draft_tokens), out.ctypes.data, ctypes.byref(st)),
           "aio_spec_generate")
    return out, {f: int(getattr(st, f)) for f, _ in aio_spec_stats._fields_}


def spec_generate(target: "DeviceModel", draft: "DeviceModel", pos: int, token: int, n_new: int,
                  k: int):
    """Draft-model speculative generation over two resident models (synchronous)."""
    # scratch of each model's own stream (the call synchronises both)
    with torch.cuda.stream(target.stream):
        tl = target.new_logits(k + 1)
        am = torch.empty(k + 1, dtype=torch.int32, device=target.device)
    with torch.cuda.stream(draft.stream):
        dl = draft.new_logits(1)
        dt = torch.empty(max(k, 1), dtype=torch.int32, device=draft.device)
    return aio_spec_generate(target.handle, draft.handle, pos, token, n_new, k, tl, dl, am, dt)


def aio_probe_route(category_logits, code_category: int, ctx_len: int, ctx_limit: int = 2048,
                    tau: float = 0.45):
    """(route to the small model?, entropy in nats, category) of the probe."""
    x = np.ascontiguousarray(category_logits, dtype=np.float32)
    h, cat = ctypes.c_float(0.0), ctypes.c_int32(-1)
    rc = lib().aio_probe_route(x.ctypes.data, int(x.size), int(code_category), int(ctx_len),
                               int(ctx_limit), float(tau), ctypes.byref(h), ctypes.byref(cat))
    if rc < 0:
        raise AioError(rc, "aio_probe_route")
    return bool(rc), float(h.value), int(cat.value)


def aio_category_entropy(handle: int, logits: torch.Tensor, label_ids, out: torch.Tensor) -> None:
    """Enqueue H(X) and the category of the label tokens' logits into out[0:2]
    (device fp32)."""
    ids = np.ascontiguousarray(label_ids, dtype=np.int32)
    _check(lib().aio_category_entropy(handle, _ptr(logits), ids.ctypes.data, int(ids.size),
                                      _ptr(out)), "aio_category_entropy")


def aio_device_status(handle: int) -> int:
    st = ctypes.c_int32(0)
    _check(lib().aio_device_status(handle, ctypes.byref(st)), "aio_device_status")
    return int(st.value)


def aio_uses_step_kernel(handle: int) -> bool:
    return bool(lib().aio_uses_step_kernel(handle))


# ------------------------------------------------- several sequences in one pool
#
# The operators below run on the current stream of their tensors' device, like
# torch's own; a tensor made or used on another stream has to be ordered with
# it by the caller, as torch asks.

_DTYPES = {torch.float32: AIO_F32, torch.bfloat16: AIO_BF16}


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _int32(*values) -> None:
    """ctypes cuts an integer to the argument's 32 bits without a word."""
    for v in values:
        if not -(1 << 31) <= v < 1 << 31:
            raise ValueError("%d does not fit 32 bits" % v)


def _host_int32(x, what: str) -> np.ndarray:
    """A host array of integers as contiguous int32, none of them cut."""
    a = np.asarray(x)
    if a.dtype != np.int32 and a.size and (  # (the search takes as long as a short call)
            a.dtype.kind not in "iu" or a.min() < -(1 << 31) or a.max() >= 1 << 31):
        raise ValueError(what + ": integers of 32 bits are needed")
    return np.ascontiguousarray(a, dtype=np.int32)


# (A decode step's calls are as short as their launches: the checks below look
# at each tensor once, and a stream is asked for as a number.)
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _packer(cls):
    """The fields of a struct to its bytes, in a quarter of the time that an
    instance of cls takes."""
    codes = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}
    s = struct.Struct("@" + "".join(codes[t] for _, t in cls._fields_) + "0q")
    assert s.size == ctypes.sizeof(cls)

    def pack(*fields) -> bytes:
        try:
            return s.pack(*fields)
        except (struct.error, OverflowError) as e:
            raise ValueError("%s: %s" % (cls.__name__, e)) from None
    return pack


(_pack_paged, _pack_packed, _pack_seqs, _pack_attn, _pack_q8, _pack_prefixes, _pack_qk) = map(
    _packer, (aio_paged_kv, aio_packed_kv, aio_seqs, aio_attn, aio_q8_kv, aio_prefixes,
              aio_qk_rows))


def _device_of(first: torch.Tensor, *others) -> int:
    """The index of the one device of the tensors (None: not given)."""
    at = first.get_device()
    _need(at >= 0, "a device tensor is needed")
    for o in others:
        if o is not None and o.get_device() != at:
            raise ValueError("tensors on different devices")
    return at


def _launch(at: int, call, *args) -> int:
    """call(*args, stream) with device ``at`` current, on its current stream."""
    if _current_device() == at:
        return call(*args, _raw_stream(at))
    with torch.cuda.device(at):
        return call(*args, _raw_stream(at))


def _i32(t: torch.Tensor, dim: int, what: str) -> None:
    if t.dtype is not torch.int32 or t.dim() != dim or (t.stride(-1) != 1 and t.numel() > 1):
        raise ValueError(what + ": an int32 tensor with %d dimension(s) is needed" % dim)


def _rows3(t: torch.Tensor, shape, what: str) -> int:
    """[rows][heads][head_dim] with the last two dimensions contiguous; its row stride."""
    n, h, d = shape
    row, head, one = t.stride()
    if (one != 1 and d > 1) or (head != d and h > 1):
        _need(t.numel() == 0, what + ": heads and dimensions have to be contiguous")
    return row if n > 1 else h * d


def _paged(k: torch.Tensor, v: torch.Tensor):
    """(aio_paged_kv's bytes, kv heads, page size, head_dim)"""
    shape, stride = k.shape, k.stride()
    if (len(shape) != 4 or v.shape != shape or k.dtype is not torch.bfloat16 or
            v.dtype is not torch.bfloat16):
        raise ValueError("pages: two bf16 [n_pages, kv_heads, page_size, head_dim]")
    pages, heads, size, hd = shape
    page_stride, head_stride, slot, one = stride
    if v.stride() != stride or one != 1 or slot != hd:
        raise ValueError("pages: K and V of the same strides, slots and dimensions contiguous")
    # (the stride of a single head or page says nothing)
    return _pack_paged(k.data_ptr(), v.data_ptr(), page_stride if pages > 1 else 0,
                       head_stride if heads > 1 else 0, pages, size, heads, hd), heads, size, hd


def _paged8(k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor):
    """(aio_q8_kv's bytes, kv heads, page size, head_dim)"""
    shape, stride = k.shape, k.stride()
    if (len(shape) != 4 or v.shape != shape or k.dtype is not torch.int8 or
            v.dtype is not torch.int8):
        raise ValueError("pages: two int8 [n_pages, kv_heads, page_size, head_dim]")
    pages, heads, size, hd = shape
    page_stride, head_stride, slot, one = stride
    if v.stride() != stride or one != 1 or slot != hd:
        raise ValueError("pages: K and V of the same strides, slots and dimensions contiguous")
    exp_shape, exp_stride = k_exp.shape, k_exp.stride()
    if (exp_shape != (pages, heads, size) or v_exp.shape != exp_shape or
            k_exp.dtype is not torch.uint8 or v_exp.dtype is not torch.uint8 or
            v_exp.stride() != exp_stride or exp_stride[2] != 1):
        raise ValueError("k_exp, v_exp: two uint8 [n_pages, kv_heads, page_size] of the same "
                         "strides, slots contiguous")
    return _pack_q8(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                    page_stride if pages > 1 else 0, head_stride if heads > 1 else 0,
                    exp_stride[0] if pages > 1 else 0, exp_stride[1] if heads > 1 else 0,
                    pages, size, heads, hd), heads, size, hd


def _prefixes(cu_seqs, prefix_lens, max_prefix, most: int) -> bytes:
    if (cu_seqs.dtype is not torch.int32 or prefix_lens.dtype is not torch.int32 or
            cu_seqs.dim() != 1 or prefix_lens.dim() != 1 or
            cu_seqs.shape[0] != prefix_lens.shape[0] + 1):
        raise ValueError("cu_seqs and prefix_lens: int32 [groups + 1] and [groups]")
    n = prefix_lens.shape[0]
    _need((n == 0 or cu_seqs.stride(0) == 1) and (n <= 1 or prefix_lens.stride(0) == 1),
          "cu_seqs and prefix_lens have to be contiguous")
    return _pack_prefixes(n, most if max_prefix is None else max_prefix, cu_seqs.data_ptr(),
                          prefix_lens.data_ptr() if n else 0)


def _paged_seqs(lens, table, cu_q, n_rows: int, max_len, page_size: int) -> bytes:
    shape = table.shape
    if (table.dtype is not torch.int32 or lens.dtype is not torch.int32 or len(shape) != 2 or
            lens.shape != shape[:1]):
        raise ValueError("lens and table: int32 [n] and [n, width]")
    n, width = shape
    row, one = table.stride()
    if n > 1:
        _need((width <= 1 or one == 1) and lens.stride(0) == 1,
              "lens and table: rows have to be contiguous")
    else:
        _need(width <= 1 or one == 1, "table: rows have to be contiguous")
        row = width
    cu = 0
    if cu_q is not None:
        if cu_q.dtype is not torch.int32 or cu_q.shape != (n + 1,) or (n and cu_q.stride(0) != 1):
            raise ValueError("cu_q: contiguous int32, one more entry than sequences")
        cu = cu_q.data_ptr()
    # (the rows of a view may lie further apart than they are wide: no key past its width)
    most = min(width * page_size, 1 << 30)
    if max_len is None or max_len > most:
        max_len = most
    return _pack_seqs(n, n_rows, max_len, cu, lens.data_ptr(), table.data_ptr(), row, 0)


def _attn(q, out, lse, scale) -> bytes:
    shape, dtype = q.shape, q.dtype
    if len(shape) != 3 or out.shape != shape or out.dtype is not dtype or dtype not in _DTYPES:
        raise ValueError("q and out: both fp32 or both bf16 [rows, heads, head_dim]")
    if lse is None:
        lse_ptr = 0
    else:
        if (lse.dtype is not torch.float32 or lse.shape != shape[:2] or
                not lse.is_contiguous()):
            raise ValueError("lse: contiguous fp32 [rows, heads]")
        lse_ptr = lse.data_ptr()
    _, heads, hd = shape
    q_stride = heads * hd if q.is_contiguous() else _rows3(q, shape, "q")
    out_stride = heads * hd if out.is_contiguous() else _rows3(out, shape, "out")
    return _pack_attn(q.data_ptr(), out.data_ptr(), lse_ptr, q_stride, out_stride, _DTYPES[dtype],
                      heads, hd ** -0.5 if scale is None else scale)


def _workspace(nbytes: int, ws, device):
    """(tensor or None, pointer) of a workspace of nbytes."""
    if nbytes == 0:
        return None, None
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    else:
        _need(ws.is_contiguous() and ws.numel() * ws.element_size() >= nbytes,
              "the workspace is smaller than %d bytes" % nbytes)
    return ws, ws.data_ptr()


def aio_attn_workspace_bytes(n_seqs: int, n_rows: int, max_len: int, n_heads: int,
                             n_kv_heads: int, head_dim: int, prompts: bool = False) -> int:
    """Workspace of an attention over n_seqs sequences with n_rows rows (prompts:
    several rows per sequence, i.e. a call with cu_q)."""
    _int32(n_seqs, n_rows, max_len, n_heads, n_kv_heads, head_dim)
    s = aio_seqs(n_seqs, n_rows, max_len, 16 if prompts else None, None, None, 0, None)
    return int(lib().aio_attn_workspace_bytes(ctypes.byref(s), n_heads, n_kv_heads, head_dim))


def _attend(call, at, kv, s, a, n_heads, n_kv_heads, head_dim, device, ws, need=None):
    n = (need or lib().aio_attn_workspace_bytes)(s, n_heads, n_kv_heads, head_dim)
    w = None
    if n:
        ws, w = _workspace(n, ws, device)
    rc = _launch(at, call, kv, s, a, w, n)
    if rc:
        raise AioError(rc, call.__name__)


def aio_paged_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor,
                        table: torch.Tensor, out: torch.Tensor, cu_q: torch.Tensor | None = None,
                        lse: torch.Tensor | None = None, scale: float | None = None,
                        max_len: int | None = None, ws: torch.Tensor | None = None) -> None:
    """Attention of q [rows, heads, head_dim] (fp32 or bf16) over the pages k, v
    (bf16 [n_pages, kv_heads, page_size, head_dim]) of the sequences with lens
    keys and table pages: one row per sequence, or with cu_q the rows of
    prompts, causal.  max_len: no sequence is longer (default: the table's
    width; a closer one gives a better split of the work)."""
    at = _device_of(q, k, v, lens, table, out, cu_q, lse, ws)
    kv, kv_heads, page_size, hd = _paged(k, v)
    a = _attn(q, out, lse, scale)
    rows, heads, q_hd = q.shape
    if q_hd != hd:
        raise ValueError("q and k differ in head_dim")
    s = _paged_seqs(lens, table, cu_q, rows, max_len, page_size)
    _attend(lib().aio_paged_attention, at, kv, s, a, heads, kv_heads, hd, q.device, ws)


def _check_heads(q, hd: int) -> None:
    if q.shape[2] != hd:
        raise ValueError("q and k differ in head_dim")


def aio_q8_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor,
                     v_exp: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
                     out: torch.Tensor, cu_q: torch.Tensor | None = None,
                     lse: torch.Tensor | None = None, scale: float | None = None,
                     max_len: int | None = None, ws: torch.Tensor | None = None) -> None:
    """aio_paged_attention over 8-bit pages: codes k, v (int8 [n_pages, kv_heads,
    page_size, head_dim]) and a byte for each row (uint8 [n_pages, kv_heads,
    page_size]), as aio_q8_append writes them."""
    at = _device_of(q, k, v, k_exp, v_exp, lens, table, out, cu_q, lse, ws)
    kv, kv_heads, page_size, hd = _paged8(k, v, k_exp, v_exp)
    a = _attn(q, out, lse, scale)
    _check_heads(q, hd)
    s = _paged_seqs(lens, table, cu_q, q.shape[0], max_len, page_size)
    L = lib()
    _attend(L.aio_q8_attention, at, kv, s, a, q.shape[1], kv_heads, hd, q.device, ws,
            L.aio_q8_workspace_bytes)


def aio_q8_workspace_bytes(n_seqs: int, n_rows: int, max_len: int, n_heads: int,
                           n_kv_heads: int, head_dim: int, prompts: bool = False) -> int:
    """Workspace of an attention over 8-bit pages, as aio_attn_workspace_bytes."""
    _int32(n_seqs, n_rows, max_len, n_heads, n_kv_heads, head_dim)
    s = aio_seqs(n_seqs, n_rows, max_len, 16 if prompts else None, None, None, 0, None)
    return int(lib().aio_q8_workspace_bytes(ctypes.byref(s), n_heads, n_kv_heads, head_dim))


def aio_prefix_workspace_bytes(n_seqs: int, n_rows: int, max_len: int, n_groups: int,
                               max_prefix: int, n_heads: int, n_kv_heads: int, head_dim: int,
                               prompts: bool = False) -> int:
    """Workspace of an attention with n_groups groups of up to max_prefix shared
    keys, otherwise as aio_attn_workspace_bytes."""
    _int32(n_seqs, n_rows, max_len, n_groups, max_prefix, n_heads, n_kv_heads, head_dim)
    s = aio_seqs(n_seqs, n_rows, max_len, 16 if prompts else None, None, None, 0, None)
    x = aio_prefixes(n_groups, max_prefix, None, None)
    return int(lib().aio_prefix_workspace_bytes(ctypes.byref(s), ctypes.byref(x), n_heads,
                                                n_kv_heads, head_dim))


def _attend_groups(call, at, kv, s, x, a, n_heads, n_kv_heads, head_dim, device, ws):
    n = lib().aio_prefix_workspace_bytes(s, x, n_heads, n_kv_heads, head_dim)
    w = None
    if n:
        ws, w = _workspace(n, ws, device)
    rc = _launch(at, call, kv, s, x, a, w, n)
    if rc:
        raise AioError(rc, call.__name__)


def aio_prefix_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor,
                         table: torch.Tensor, cu_seqs: torch.Tensor, prefix_lens: torch.Tensor,
                         out: torch.Tensor, cu_q: torch.Tensor | None = None,
                         lse: torch.Tensor | None = None, scale: float | None = None,
                         max_len: int | None = None, max_prefix: int | None = None,
                         ws: torch.Tensor | None = None) -> None:
    """aio_paged_attention of sequences in groups: those from cu_seqs[g] up to
    cu_seqs[g + 1] begin with the same prefix_lens[g] keys, which are read once for all
    of them.  max_prefix: no prefix is longer (default: max_len; state it closely where
    sequences have many keys beyond their prefixes, which are split by the difference)."""
    at = _device_of(q, k, v, lens, table, cu_seqs, prefix_lens, out, cu_q, lse, ws)
    kv, kv_heads, page_size, hd = _paged(k, v)
    a = _attn(q, out, lse, scale)
    _check_heads(q, hd)
    s = _paged_seqs(lens, table, cu_q, q.shape[0], max_len, page_size)
    x = _prefixes(cu_seqs, prefix_lens, max_prefix, 1 << 30)
    _attend_groups(lib().aio_prefix_attention, at, kv, s, x, a, q.shape[1], kv_heads, hd,
                   q.device, ws)


def aio_q8_prefix_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                            k_exp: torch.Tensor, v_exp: torch.Tensor, lens: torch.Tensor,
                            table: torch.Tensor, cu_seqs: torch.Tensor,
                            prefix_lens: torch.Tensor, out: torch.Tensor,
                            cu_q: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                            scale: float | None = None, max_len: int | None = None,
                            max_prefix: int | None = None,
                            ws: torch.Tensor | None = None) -> None:
    """aio_prefix_attention over the 8-bit pages of aio_q8_attention."""
    at = _device_of(q, k, v, k_exp, v_exp, lens, table, cu_seqs, prefix_lens, out, cu_q, lse, ws)
    kv, kv_heads, page_size, hd = _paged8(k, v, k_exp, v_exp)
    a = _attn(q, out, lse, scale)
    _check_heads(q, hd)
    s = _paged_seqs(lens, table, cu_q, q.shape[0], max_len, page_size)
    x = _prefixes(cu_seqs, prefix_lens, max_prefix, 1 << 30)
    _attend_groups(lib().aio_q8_prefix_attention, at, kv, s, x, a, q.shape[1], kv_heads, hd,
                   q.device, ws)


def aio_packed_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor,
                         cu_k: torch.Tensor, out: torch.Tensor, lse: torch.Tensor | None = None,
                         scale: float | None = None, max_len: int | None = None,
                         ws: torch.Tensor | None = None) -> None:
    """Causal attention of the packed rows q over packed keys and values k, v
    (bf16 [keys, kv_heads, head_dim]); cu_q and cu_k give each sequence's first
    row and key."""
    at = _device_of(q, k, v, cu_q, cu_k, out, lse, ws)
    a = _attn(q, out, lse, scale)
    _need(k.dim() == 3 and k.shape == v.shape and k.dtype == v.dtype == torch.bfloat16 and
          k.shape[2] == q.shape[2], "k, v: two bf16 [keys, kv_heads, head_dim]")
    _need(k.stride() == v.stride() and (k.numel() == 0 or k.stride(2) == 1),
          "k, v: the same strides, dimensions contiguous")
    for t, what in ((cu_q, "cu_q"), (cu_k, "cu_k")):
        _i32(t, 1, what)
    _need(cu_q.shape == cu_k.shape and cu_q.shape[0] >= 1, "cu_q and cu_k differ in length")
    rows, heads, hd = k.shape
    kv = _pack_packed(k.data_ptr(), v.data_ptr(), k.stride(0) if rows > 1 else 0,
                      k.stride(1) if heads > 1 else 0, rows, heads, hd)
    s = _pack_seqs(cu_q.shape[0] - 1, q.shape[0], rows if max_len is None else max_len,
                   cu_q.data_ptr(), 0, 0, 0, cu_k.data_ptr())
    _attend(lib().aio_packed_attention, at, kv, s, a, q.shape[1], heads, hd, q.device, ws)


def aio_page_append(k_rows: torch.Tensor, v_rows: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                    lens: torch.Tensor, table: torch.Tensor, cu_q: torch.Tensor | None = None,
                    max_len: int | None = None) -> None:
    """Write the new rows' keys and values ([rows, kv_heads, head_dim], fp32 or
    bf16) into their pages; lens counts them already."""
    at = _device_of(k, v, k_rows, v_rows, lens, table, cu_q)
    kv, kv_heads, page_size, hd = _paged(k, v)
    _append(lib().aio_page_append, at, kv, kv_heads, page_size, hd, k_rows, v_rows, lens, table,
            cu_q, max_len)


def aio_q8_append(k_rows: torch.Tensor, v_rows: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                  k_exp: torch.Tensor, v_exp: torch.Tensor, lens: torch.Tensor,
                  table: torch.Tensor, cu_q: torch.Tensor | None = None,
                  max_len: int | None = None) -> None:
    """aio_page_append into the 8-bit pages of aio_q8_attention: each head's row
    becomes int8 codes and the byte of their power of two."""
    at = _device_of(k, v, k_exp, v_exp, k_rows, v_rows, lens, table, cu_q)
    kv, kv_heads, page_size, hd = _paged8(k, v, k_exp, v_exp)
    _append(lib().aio_q8_append, at, kv, kv_heads, page_size, hd, k_rows, v_rows, lens, table,
            cu_q, max_len)


def _append(call, at, kv, kv_heads, page_size, hd, k_rows, v_rows, lens, table, cu_q, max_len):
    shape, stride, dtype = k_rows.shape, k_rows.stride(), k_rows.dtype
    if (len(shape) != 3 or v_rows.shape != shape or v_rows.dtype is not dtype or
            dtype not in _DTYPES or shape[1] != kv_heads or shape[2] != hd):
        raise ValueError("rows: two fp32 or bf16 [rows, kv_heads, head_dim]")
    if v_rows.stride() != stride or stride[2] != 1:
        _need(k_rows.numel() == 0, "rows: the same strides, dimensions contiguous")
    s = _paged_seqs(lens, table, cu_q, shape[0], max_len, page_size)
    rc = _launch(at, call, kv, s, k_rows.data_ptr(), v_rows.data_ptr(), _DTYPES[dtype],
                 stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0)
    if rc:
        raise AioError(rc, call.__name__)


def _head_weight(w: torch.Tensor, hd: int) -> int:
    if w.dtype is not torch.bfloat16 or w.shape != (hd,) or (w.stride(0) != 1 and hd > 1):
        raise ValueError("q_weight, k_weight: contiguous bf16 [head_dim]")
    return w.data_ptr()


def aio_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor,
                     q_out: torch.Tensor, k_out: torch.Tensor,
                     q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
                     eps: float = 1e-5, base: float = 10000.0) -> None:
    """RMS norm of each head of q [rows, heads, head_dim] and k [rows, kv_heads,
    head_dim] (both fp32 or bf16), times the weights (bf16 [head_dim], None: 1), and the
    rotation of its halves by the row's position (int32).  An output may be its input."""
    at = _device_of(q, k, positions, q_out, k_out, q_weight, k_weight)
    shape, k_shape, dtype = q.shape, k.shape, q.dtype
    if (len(shape) != 3 or len(k_shape) != 3 or k_shape[0] != shape[0] or
            k_shape[2] != shape[2] or dtype not in _DTYPES or k.dtype is not dtype or
            q_out.shape != shape or k_out.shape != k_shape or q_out.dtype is not dtype or
            k_out.dtype is not dtype):
        raise ValueError("q, k and their outputs: all fp32 or all bf16 [rows, heads, head_dim]")
    rows, heads, hd = shape
    _i32(positions, 1, "positions")
    _need(positions.shape[0] == rows, "one position per row")
    qw = kw = None
    if q_weight is not None:
        qw = _head_weight(q_weight, hd)
    if k_weight is not None:
        kw = _head_weight(k_weight, hd)
    r = _pack_qk(q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(),
                 _rows3(q, shape, "q"), _rows3(k, k_shape, "k"), _rows3(q_out, shape, "q_out"),
                 _rows3(k_out, k_shape, "k_out"), _DTYPES[dtype], rows, heads, k_shape[1], hd)
    rc = _launch(at, lib().aio_qk_norm_rope, r, positions.data_ptr(), qw, kw, eps, base)
    if rc:
        raise AioError(rc, "aio_qk_norm_rope")


def aio_page_copy(pool: torch.Tensor, src, dst) -> None:
    """Copy pages src[i] to dst[i] (host int32 arrays) in every plane of the pool
    [planes, n_pages, ...], whose pages are contiguous."""
    at = _device_of(pool)
    shape, stride, inner = pool.shape, pool.stride(), 1
    _need(len(shape) >= 3 and pool.numel() > 0, "pool: [planes, n_pages, ...]")
    for n, st in zip(shape[:1:-1], stride[:1:-1]):
        _need(n == 1 or st == inner, "pool: pages have to be contiguous")
        inner *= n
    a, b = _host_int32(src, "src"), _host_int32(dst, "dst")
    _int32(shape[0], shape[1], a.size)
    _need(a.ndim == 1 and a.shape == b.shape, "src and dst differ in length")
    size = pool.element_size()
    rc = _launch(at, lib().aio_page_copy, pool.data_ptr(), shape[0], stride[0] * size, shape[1],
                 (stride[1] if shape[1] > 1 else inner) * size, inner * size, a.ctypes.data,
                 b.ctypes.data, a.size)
    if rc:
        raise AioError(rc, "aio_page_copy")


def aio_logprobs_workspace_bytes(rows: int, n: int, top: int) -> int:
    _int32(rows, n, top)
    return int(lib().aio_logprobs_workspace_bytes(rows, n, top))


def aio_logprobs(logits: torch.Tensor, targets: torch.Tensor | None,
                 logprob: torch.Tensor | None, entropy: torch.Tensor | None,
                 top_ids: torch.Tensor | None = None, top_logprobs: torch.Tensor | None = None,
                 ws: torch.Tensor | None = None) -> None:
    """Log probabilities of the targets, entropies and the top alternatives of
    logits [rows, n] (fp32 or bf16); each output may be None."""
    at = _device_of(logits, targets, logprob, entropy, top_ids, top_logprobs, ws)
    dtype = logits.dtype
    _need(logits.dim() == 2 and dtype in _DTYPES, "logits: fp32 or bf16 [rows, n]")
    rows, n = logits.shape
    _int32(rows, n)
    _need(n <= 1 or rows == 0 or logits.stride(1) == 1, "logits: rows have to be contiguous")
    if targets is not None:
        _i32(targets, 1, "targets")
        _need(targets.shape[0] == rows, "one target per row")
    for t in (logprob, entropy):
        if t is not None and (t.dtype is not torch.float32 or t.shape != (rows,) or
                              not t.is_contiguous()):
            raise ValueError("logprob, entropy: contiguous fp32 [rows]")
    _need((top_ids is None) == (top_logprobs is None), "top_ids and top_logprobs go together")
    top = 0
    if top_ids is not None:
        _i32(top_ids, 2, "top_ids")
        top = top_ids.shape[1]
        if (top_ids.shape[0] != rows or top_logprobs.shape != top_ids.shape or
                top_logprobs.dtype is not torch.float32 or not top_ids.is_contiguous() or
                not top_logprobs.is_contiguous()):
            raise ValueError("top_ids, top_logprobs: contiguous int32 and fp32 [rows, top]")
    L = lib()
    need = L.aio_logprobs_workspace_bytes(rows, n, top)
    ws, w = _workspace(need, ws, logits.device)
    rc = _launch(at, L.aio_logprobs, logits.data_ptr(), _DTYPES[dtype], rows, n,
                 logits.stride(0) if rows > 1 else n, _ptr(targets), top, _ptr(logprob),
                 _ptr(entropy), _ptr(top_ids), _ptr(top_logprobs), w, need)
    if rc:
        raise AioError(rc, "aio_logprobs")


class Pages:
    """Which pages of a pool each sequence holds (host bookkeeping: aio_pages_*).
    ``extend`` and ``compact`` return the copies (src, dst) to enqueue."""

    def __init__(self, n_pages: int, page_size: int, max_seqs: int):
        _int32(n_pages, page_size, max_seqs)
        h = ctypes.c_void_p()
        _check(lib().aio_pages_create(n_pages, page_size, max_seqs, ctypes.byref(h)),
               "aio_pages_create")
        self.handle, self.n_pages, self.page_size = h.value, n_pages, page_size

    def open(self) -> int:
        s = ctypes.c_int32(-1)
        _check(lib().aio_pages_open(self.handle, ctypes.byref(s)), "aio_pages_open")
        return s.value

    def close(self, seq: int) -> None:
        _int32(seq)
        _check(lib().aio_pages_close(self.handle, seq), "aio_pages_close")

    def fork(self, seq: int) -> int:
        _int32(seq)
        s = ctypes.c_int32(-1)
        _check(lib().aio_pages_fork(self.handle, seq, ctypes.byref(s)), "aio_pages_fork")
        return s.value

    def extend(self, seq: int, n: int):
        _int32(seq, n)
        a, b, c = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
        _check(lib().aio_pages_extend(self.handle, seq, n, ctypes.byref(a), ctypes.byref(b),
                                      ctypes.byref(c)), "aio_pages_extend")
        return ([a.value], [b.value]) if c.value else ([], [])

    def truncate(self, seq: int, length: int) -> None:
        _int32(seq, length)
        _check(lib().aio_pages_truncate(self.handle, seq, length), "aio_pages_truncate")

    def compact(self):
        a, b = np.empty(self.n_pages, np.int32), np.empty(self.n_pages, np.int32)
        n = ctypes.c_int32(0)
        _check(lib().aio_pages_compact(self.handle, a.ctypes.data, b.ctypes.data, self.n_pages,
                                       ctypes.byref(n)), "aio_pages_compact")
        return a[: n.value].copy(), b[: n.value].copy()

    def length(self, seq: int) -> int:
        _int32(seq)
        n = ctypes.c_int32(0)
        _check(lib().aio_pages_row(self.handle, seq, None, 0, ctypes.byref(n)), "aio_pages_row")
        return n.value

    def rows(self, seqs, width: int):
        """(lens [n], table [n, width]) of the sequences, host int32."""
        _int32(width, *seqs)
        lens, table = np.zeros(len(seqs), np.int32), np.full((len(seqs), width), -1, np.int32)
        n = ctypes.c_int32(0)
        for i, s in enumerate(seqs):
            _check(lib().aio_pages_row(self.handle, s, table[i].ctypes.data, width,
                                       ctypes.byref(n)), "aio_pages_row")
            lens[i] = n.value
        return lens, table

    @property
    def free(self) -> int:
        return int(lib().aio_pages_free(self.handle))

    def destroy(self) -> None:
        if getattr(self, "handle", None):
            lib().aio_pages_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ------------------------------------------------------------------ a model

def _to_device(a: np.ndarray, device) -> torch.Tensor:
    if a.dtype == np.uint16:
        t = torch.from_numpy(a.view(np.int16)).to(device)
        return t.view(torch.bfloat16)
    if a.dtype == np.int8:
        return torch.from_numpy(a).to(device)
    raise TypeError(a.dtype)


class DeviceModel:
    """Weights, KV cache and workspace in device memory plus a loaded handle.

    ``weights`` maps tensor names (``embed``, ``final_norm``, ``lm_head``,
    ``layers.{l}.{attn_norm, ffn_norm, wq, ...}``, ``*.scale``) to numpy
    arrays of storage bits; they are copied to the device once."""

    def __init__(self, cfg, weights: dict, kv_init: np.ndarray | None = None,
                 device: str = "cuda:0", stream: torch.cuda.Stream | None = None):
        self.cfg = cfg
        self.c = make_config(cfg)
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        int8 = self.c.wfmt == AIO_WFMT_INT8
        self.dev = {k: _to_device(v, self.device) for k, v in weights.items()}
        kvb, wsb = aio_kv_bytes(self.c), aio_workspace_bytes(self.c)
        if kvb == 0 or wsb == 0:
            raise AioError(aio_check_config(self.c), "config")
        if kv_init is not None:
            assert kv_init.nbytes == kvb and kv_init.dtype == np.uint16
            self.kv = _to_device(np.ascontiguousarray(kv_init).reshape(-1), self.device)
        else:
            self.kv = torch.zeros(kvb // 2, dtype=torch.bfloat16, device=self.device)
        self.ws = torch.zeros(wsb, dtype=torch.uint8, device=self.device)
        layers = (aio_layer_weights * self.c.n_layers)()
        for l in range(self.c.n_layers):
            p = "layers.%d." % l
            L = layers[l]
            L.attn_norm = _ptr(self.dev[p + "attn_norm"])
            L.ffn_norm = _ptr(self.dev[p + "ffn_norm"])
            for n, s in zip(LINEARS, SCALES):
                setattr(L, n, _ptr(self.dev[p + n]))
                setattr(L, s, _ptr(self.dev[p + n + ".scale"]) if int8 else None)
        self._layers = layers
        w = aio_weights()
        w.embed = _ptr(self.dev["embed"])
        w.final_norm = _ptr(self.dev["final_norm"])
        w.lm_head = _ptr(self.dev["lm_head"])
        w.s_lm_head = _ptr(self.dev["lm_head.scale"]) if int8 else None
        w.layers = ctypes.cast(layers, ctypes.POINTER(aio_layer_weights))
        self._w = w
        torch.cuda.synchronize(self.device)
        self.handle = aio_model_load(self.c, w, self.kv, self.ws, self.stream.cuda_stream)

    def kv_numpy(self) -> np.ndarray:
        """The device KV cache as uint16 bf16 bits in the oracle's layout."""
        c = self.c
        t = self.kv.view(torch.int16).cpu().numpy().view(np.uint16)
        return t.reshape(c.n_layers, 2, c.n_kv_heads, c.max_ctx, c.head_dim)

    def kv_rows(self, lo: int, hi: int) -> np.ndarray:
        """Cache positions [lo, hi) as uint16 bf16 bits, [layer, K/V, kv head,
        position, head_dim] (only those rows cross to the host)."""
        c = self.c
        t = self.kv.view(torch.int16).view(c.n_layers, 2, c.n_kv_heads, c.max_ctx, c.head_dim)
        return t[:, :, :, lo:hi, :].cpu().numpy().view(np.uint16)

    def new_logits(self, rows: int = 1) -> torch.Tensor:
        return torch.empty((rows, self.c.vocab), dtype=torch.float32, device=self.device)

    def decode_step(self, token: int, pos: int, logits: torch.Tensor) -> None:
        aio_decode_step(self.handle, token, pos, logits)

    def verify(self, token: int, drafts, pos: int, logits: torch.Tensor) -> None:
        aio_verify(self.handle, token, drafts, len(drafts), pos, logits)

    def argmax(self, logits: torch.Tensor, rows: int, out: torch.Tensor) -> None:
        aio_argmax(self.handle, logits, rows, logits.shape[-1], out)

    def greedy(self, token: int, pos: int, n_steps: int, tokens: torch.Tensor,
               logits: torch.Tensor) -> None:
        aio_decode_greedy(self.handle, token, pos, n_steps, tokens, logits)

    def pld_generate(self, history, pos: int, token: int, n_new: int, ngram_max: int,
                     ngram_min: int, k: int):
        """Prompt-lookup greedy generation of n_new tokens (synchronous)."""
        with torch.cuda.stream(self.stream):
            logits = self.new_logits(k + 1)
            am = torch.empty(k + 1, dtype=torch.int32, device=self.device)
        return aio_pld_generate(self.handle, history, pos, token, n_new, ngram_max, ngram_min, k,
                                logits, am)

    def prefill(self, tokens, pos: int, logits: torch.Tensor) -> None:
        """Consume tokens at pos.. in prompt-length matrix products; logits
        (fp32, at least [vocab]) receives the last token's logits."""
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        _check(lib().aio_prefill(self.handle, t.ctypes.data, int(t.size), int(pos), _ptr(logits)),
               "aio_prefill")

    def prefill_noalloc(self, tokens, pos: int, logits: torch.Tensor) -> None:
        """aio_prefill with the scratch in the library's fixed device array
        (no device allocation)."""
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        _check(lib().aio_prefill_noalloc(self.handle, t.ctypes.data, int(t.size), int(pos),
                                         _ptr(logits)), "aio_prefill_noalloc")

    @property
    def prefill_noalloc_rows(self) -> int:
        return int(lib().aio_prefill_noalloc_rows(ctypes.byref(self.c)))

    def new_pool(self, n_pages: int, page_size: int = 16) -> torch.Tensor:
        """A paged cache for this model: bf16 [layer, K/V, page, kv head, slot, dim]."""
        c = self.c
        return torch.zeros((c.n_layers, 2, n_pages, c.n_kv_heads, page_size, c.head_dim),
                           dtype=torch.bfloat16, device=self.device)

    def paged_forward(self, pool: torch.Tensor, rows, lens, table, tokens, out_rows,
                      logits: torch.Tensor) -> None:
        """One pass over the next tokens of several sequences in ``pool`` (a
        new_pool tensor): rows[i] tokens of sequence i, which then has lens[i]
        and the pages table[i] (host arrays).  logits [len(out_rows), vocab]
        receives those of the packed rows out_rows.  On the model's stream."""
        c = self.c
        _need(pool.dim() == 6 and pool.dtype == torch.bfloat16 and pool.is_contiguous() and
              pool.shape[:2] == (c.n_layers, 2),
              "pool: a contiguous bf16 [layers, 2, n_pages, kv_heads, page_size, head_dim]")
        device = self.kv.device  # (which "cuda" alone does not name)
        _need(pool.device == device and logits.device == device,
              "pool and logits: on the model's device")
        a = [_host_int32(x, what) for x, what in (
            (rows, "rows"), (lens, "lens"), (table, "table"), (tokens, "tokens"),
            (out_rows, "out_rows"))]
        n = a[0].size
        _need(a[1].size == n and a[2].ndim == 2 and a[2].shape[0] == n and
              a[3].size == a[0].sum(dtype=np.int64), "rows, lens, table and tokens do not match")
        _need(logits.dtype == torch.float32 and logits.is_contiguous() and
              logits.numel() >= a[4].size * c.vocab, "logits: contiguous fp32 [out rows, vocab]")
        kv = aio_paged_kv(pool.data_ptr(), pool[0, 1].data_ptr(), pool.stride(2), pool.stride(3),
                          pool.shape[2], pool.shape[4], pool.shape[3], pool.shape[5])
        p = aio_paged_pool(kv, pool.stride(0), pool.shape[0])
        need = int(lib().aio_paged_forward_bytes(ctypes.byref(c), n, int(a[3].size),
                                                 a[2].shape[1]))
        with torch.cuda.device(device), torch.cuda.stream(self.stream):
            if getattr(self, "_paged_scratch", None) is None or \
                    self._paged_scratch.numel() < need:
                self._paged_scratch = torch.empty(max(need, 256), dtype=torch.uint8,
                                                  device=device)
            s = self._paged_scratch
            _check(lib().aio_paged_forward(self.handle, ctypes.byref(p), n, a[0].ctypes.data,
                                           a[1].ctypes.data, a[2].ctypes.data, a[2].shape[1],
                                           a[3].ctypes.data, a[4].ctypes.data, int(a[4].size),
                                           _ptr(logits), s.data_ptr(), s.numel()),
                   "aio_paged_forward")

    def tune(self, token: int, pos: int, logits: torch.Tensor, rounds: int = 4) -> None:
        """Calibrate the persistent kernel's gate/up split (aio_tune_step)."""
        _check(lib().aio_tune_step(self.handle, int(token), int(pos), _ptr(logits), int(rounds)),
               "aio_tune_step")

    def profile_step(self, token: int, pos: int, logits: torch.Tensor) -> np.ndarray:
        return aio_profile_step(self.handle, token, pos, logits, 6 * self.c.n_layers + 1)

    def trace_step(self, token: int, pos: int, logits: torch.Tensor) -> np.ndarray:
        return aio_trace_step(self.handle, token, pos, logits, 5 * self.c.n_layers + 1)

    @property
    def uses_step_kernel(self) -> bool:
        return aio_uses_step_kernel(self.handle)

    def status(self) -> int:
        """Device-side status word (0 = fine); synchronises."""
        return aio_device_status(self.handle)

    def sync(self) -> None:
        self.stream.synchronize()

    def close(self) -> None:
        if getattr(self, "handle", None):
            aio_model_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
