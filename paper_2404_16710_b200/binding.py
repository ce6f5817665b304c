"""Thin ctypes binding of the C ABI in ``include/ls.h`` -- argument marshalling only.

Every function has the name of the C entry point it calls.  Device operands are torch
CUDA tensors (only their ``data_ptr()`` crosses the boundary), host operands are numpy
arrays.  PyTorch is used for device memory and streams, nothing else: every step of the
path runs in the library's own kernels.  There is no fallback: if ``libls_b200.so`` is
missing the first call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
from pathlib import Path

import numpy as np

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libls_b200.so"

LS_OK = 0
LS_ERR_INVALID_ARG, LS_ERR_CAPACITY, LS_ERR_CUDA, LS_ERR_DEVICE_STATUS, LS_ERR_UNSUPPORTED = -1, -2, -3, -4, -5
LS_MAX_ROWS = 16
LS_LINEAR_AUTO, LS_LINEAR_FMA, LS_LINEAR_MMA = 0, 1, 2

EXPORTS = (
    "ls_strerror", "ls_last_cuda_error", "ls_workspace_bytes", "ls_model_create", "ls_model_destroy",
    "ls_set_page_table", "ls_generate", "ls_generate_adaptive", "ls_generate_full", "ls_generate_early", "ls_prefill",
    "ls_decode", "ls_decode_flags", "ls_decode_adaptive", "ls_read_output", "ls_read_drafted",
    "ls_generate_batch", "ls_prefill_batch", "ls_decode_batch", "ls_read_output_seq", "ls_debug_logits", "ls_debug_next_logits", "ls_get_stats", "ls_op_embed", "ls_op_rmsnorm",
    "ls_op_linear", "ls_op_gate_up_swiglu", "ls_op_lm_head_scratch_bytes", "ls_op_lm_head_argmax",
    "ls_op_lm_head_argmax_static", "ls_op_rope_append", "ls_op_qkv_rope_append", "ls_op_attention", "ls_op_accept",
    "ls_op_gemm", "ls_op_prefill_attention", "ls_op_chain", "ls_op_w4_bytes", "ls_op_quantize_w4", "ls_op_expand_w4",
    "ls_op_linear_w4", "ls_op_kv4_page_bytes", "ls_op_append_kv4", "ls_op_expand_kv4", "ls_op_attention_kv4",
    "ls_op_attention_kv4_scratch_bytes", "ls_op_f8_scale_bytes", "ls_op_quantize_f8", "ls_op_expand_f8", "ls_op_rmsnorm_f8",
    "ls_op_swiglu_f8", "ls_op_linear_f8",
)


class LsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().ls_strerror(status).decode()
        if status == LS_ERR_CUDA:
            msg += f" [cudaError {lib().ls_last_cuda_error()}]"
        super().__init__(f"{where}: {msg} ({status})")


class ls_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ffn", C.c_int32),
                ("vocab", C.c_int32), ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("max_seq", C.c_int32), ("page_size", C.c_int32), ("max_draft", C.c_int32),
                ("eos_id", C.c_int32), ("linear_path", C.c_int32)]


_VPP = C.POINTER(C.c_void_p)


class ls_weights(C.Structure):
    _fields_ = [("tok_embed", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)] + \
               [(n, _VPP) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class ls_stats(C.Structure):
    _fields_ = [("prefill_ms", C.c_double), ("decode_ms", C.c_double), ("weight_bytes", C.c_int64),
                ("kv_bytes", C.c_int64), ("kernel_launches", C.c_int64), ("n_generated", C.c_int32),
                ("n_steps", C.c_int32), ("n_accepted", C.c_int32), ("host_syncs", C.c_int32)]


_lib = None


def lib():
    """Load the CUDA library (built in-tree by ``paper_2404_16710_b200.build``)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2404_16710_b200.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(str(LIB_PATH))
        i64 = C.c_int64
        i32, vp, ip, fp = C.c_int32, C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_float)
        sig = {
            "ls_strerror": (C.c_char_p, [C.c_int]),
            "ls_last_cuda_error": (C.c_int, []),
            "ls_workspace_bytes": (C.c_size_t, [C.POINTER(ls_config)]),
            "ls_model_create": (C.c_int, [C.POINTER(ls_config), C.POINTER(ls_weights), vp, C.c_size_t, vp,
                                          C.POINTER(vp)]),
            "ls_model_destroy": (C.c_int, [vp]),
            "ls_set_page_table": (C.c_int, [vp, ip, i32]),
            "ls_generate": (C.c_int, [vp, ip, i32, i32, i32, i32, ip, ip, ip, ip]),
            "ls_generate_full": (C.c_int, [vp, ip, i32, i32, ip, ip]),
            "ls_generate_early": (C.c_int, [vp, ip, i32, i32, i32, ip, ip]),
            "ls_prefill": (C.c_int, [vp, ip, i32, i32]),
            "ls_decode": (C.c_int, [vp, i32, i32, i32]),
            "ls_decode_flags": (C.c_int, [vp, i32, i32, i32, i32]),
            "ls_read_output": (C.c_int, [vp, ip, ip, ip, ip]),
            "ls_generate_batch": (C.c_int, [vp, i32, ip, ip, i32, i32, i32, ip, ip, ip, ip]),
            "ls_prefill_batch": (C.c_int, [vp, i32, ip, ip]),
            "ls_decode_batch": (C.c_int, [vp, i32, i32, i32]),
            "ls_read_output_seq": (C.c_int, [vp, i32, ip, ip, ip, ip]),
            "ls_generate_adaptive": (C.c_int, [vp, ip, i32, i32, i32, C.c_float, i32, ip, ip, ip, ip, ip]),
            "ls_decode_adaptive": (C.c_int, [vp, i32, i32, C.c_float, i32]),
            "ls_read_drafted": (C.c_int, [vp, ip, ip]),
            "ls_debug_logits": (C.c_int, [vp, ip, i32, i32, fp, fp]),
            "ls_debug_next_logits": (C.c_int, [vp, fp]),
            "ls_get_stats": (C.c_int, [vp, C.POINTER(ls_stats)]),
            "ls_op_chain": (C.c_int, [i32]),
            "ls_op_embed": (C.c_int, [vp, vp, i32, i32, i32, vp, vp]),
            "ls_op_rmsnorm": (C.c_int, [vp, vp, i32, i32, C.c_float, vp, vp]),
            "ls_op_linear": (C.c_int, [i32, vp, vp, i32, i32, i32, vp, i32, vp]),
            "ls_op_gate_up_swiglu": (C.c_int, [i32, vp, vp, vp, i32, i32, i32, vp, vp]),
            "ls_op_lm_head_scratch_bytes": (C.c_size_t, [i32]),
            "ls_op_lm_head_argmax": (C.c_int, [i32, vp, vp, i32, i32, i32, vp, vp, vp, vp]),
            "ls_op_lm_head_argmax_static": (C.c_int, [i32, vp, vp, i32, i32, i32, vp, vp]),
            "ls_op_rope_append": (C.c_int, [vp, i32, i32, i32, i32, i32, C.c_float, i32, vp, i32, vp, vp, vp, vp]),
            "ls_op_qkv_rope_append": (C.c_int, [i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, C.c_float, i32, vp, i32,
                                                vp, vp, vp, vp]),
            "ls_op_attention": (C.c_int, [vp, i32, i32, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp]),
            "ls_op_accept": (C.c_int, [vp, vp, i32, vp, vp, vp, vp]),
            "ls_op_gemm": (C.c_int, [vp, vp, i32, i32, i32, vp, i32, i32, vp, vp]),
            "ls_op_prefill_attention": (C.c_int, [vp, i32, i32, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp]),
            "ls_op_w4_bytes": (C.c_size_t, [i32, i32, i32]),
            "ls_op_quantize_w4": (C.c_int, [vp, i32, i32, i32, vp, vp]),
            "ls_op_expand_w4": (C.c_int, [vp, i32, i32, i32, vp, vp]),
            "ls_op_linear_w4": (C.c_int, [vp, vp, i32, i32, i32, i32, vp, i32, vp]),
            "ls_op_kv4_page_bytes": (C.c_size_t, [i32, i32, i32]),
            "ls_op_append_kv4": (C.c_int, [vp, vp, i64, i64, i64, i32, i32, vp, i32, i32, i32, vp, i32, i32, vp, i32, vp, vp]),
            "ls_op_expand_kv4": (C.c_int, [vp, i32, i32, i32, vp, i32, i32, i32, vp, i32, i32, vp, vp, vp, i32, vp, vp]),
            "ls_op_attention_kv4": (C.c_int, [vp, i32, i32, vp, i32, i32, i32, i32, vp, i32, i32, vp, i32, vp, vp, vp, vp]),
            "ls_op_attention_kv4_scratch_bytes": (C.c_size_t, [i32, i32, i32, i32, i32, i32]),
            "ls_op_f8_scale_bytes": (C.c_size_t, [i32, i32, i32]),
            "ls_op_quantize_f8": (C.c_int, [vp, i32, i64, i32, i32, i32, vp, vp, vp]),
            "ls_op_expand_f8": (C.c_int, [vp, vp, i32, i32, i32, vp, vp]),
            "ls_op_rmsnorm_f8": (C.c_int, [vp, i32, i64, vp, i32, i64, vp, i64, vp, i32, i32, C.c_float, vp, vp, vp]),
            "ls_op_swiglu_f8": (C.c_int, [vp, vp, i32, i64, i32, i32, vp, vp, vp]),
            "ls_op_linear_f8": (C.c_int, [vp, vp, vp, vp, i32, i32, i32, vp, i32, i64, vp, i64, vp, vp]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _ck(rc, where):
    if rc != LS_OK:
        raise LsError(rc, where)


def _dev(t):
    """device pointer of a torch CUDA tensor (None -> NULL)"""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    return C.c_void_p(t.data_ptr())


class _Torch:
    """what the single operations need of torch, looked up once: a call of a few microseconds notices"""

    def load(self):
        import torch
        self.bf16, self.f32, self.i32, self.u8, self.empty = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.empty
        self.f8 = torch.float8_e4m3fn
        # torch.cuda.current_stream() builds a Stream object (3.4 us a call, as much as a launch); the raw handle costs 0.2
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.stream = raw or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        self.device = torch.cuda.current_device
        return self

    def __getattr__(self, name):  # only before load()
        return getattr(self.load(), name)


_torch = _Torch()


def _stream():
    """handle of the current CUDA stream"""
    return _torch.stream(_torch.device())


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


# ------------------------------------------------------------------ model-level entry points
def make_config(shape, max_seq, page_size=64, max_draft=8, eos_id=-1, linear_path=LS_LINEAR_AUTO) -> ls_config:
    """shape: any object with the decoder-shape attributes (e.g. synth.Shape)."""
    return ls_config(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.head_dim,
                     shape.d_ffn, shape.vocab, shape.rms_eps, shape.rope_theta, max_seq, page_size,
                     max_draft, eos_id, linear_path)


def ls_workspace_bytes(cfg: ls_config) -> int:
    return lib().ls_workspace_bytes(C.byref(cfg))


def ls_model_create(cfg: ls_config, weights: dict, workspace, stream=None):
    """weights: dict of torch bf16 CUDA tensors (per-layer entries are lists).  Returns the
    opaque handle; the caller keeps ``weights`` and ``workspace`` alive."""
    w = ls_weights()
    keep = []
    for k in ("tok_embed", "final_norm", "lm_head"):
        setattr(w, k, weights[k].data_ptr())
    for k in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"):
        arr = (C.c_void_p * cfg.n_layers)(*[t.data_ptr() for t in weights[k]])
        keep.append(arr)
        setattr(w, k, C.cast(arr, _VPP))
    h = C.c_void_p()
    st = C.c_void_p(stream) if stream else None  # None: the model makes a stream of its own
    _ck(lib().ls_model_create(C.byref(cfg), C.byref(w), _dev(workspace), workspace.numel() * workspace.element_size(),
                              st, C.byref(h)), "ls_model_create")
    return h


def ls_model_destroy(h):
    _ck(lib().ls_model_destroy(h), "ls_model_destroy")


def ls_set_page_table(h, table):
    a, p = _i32(table)
    _ck(lib().ls_set_page_table(h, p, a.size), "ls_set_page_table")


def ls_generate(h, prompt, exit_layer, num_draft, max_new):
    """-> (ids, accepted_per_step) as numpy int32 arrays"""
    a, p = _i32(prompt)
    out, acc = np.zeros(max_new, np.int32), np.zeros(max_new, np.int32)
    n, s = C.c_int32(), C.c_int32()
    _ck(lib().ls_generate(h, p, a.size, exit_layer, num_draft, max_new,
                          out.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(n),
                          acc.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(s)), "ls_generate")
    return out[:n.value], acc[:s.value]


def ls_generate_adaptive(h, prompt, exit_layer, max_draft, min_margin, max_new):
    """-> (ids, accepted_per_step, drafted_per_step) as numpy int32 arrays"""
    a, p = _i32(prompt)
    out, acc, dr = np.zeros(max_new, np.int32), np.zeros(max_new, np.int32), np.zeros(max_new, np.int32)
    n, s = C.c_int32(), C.c_int32()
    ip = C.POINTER(C.c_int32)
    _ck(lib().ls_generate_adaptive(h, p, a.size, exit_layer, max_draft, float(min_margin), max_new,
                                   out.ctypes.data_as(ip), C.byref(n), acc.ctypes.data_as(ip),
                                   dr.ctypes.data_as(ip), C.byref(s)), "ls_generate_adaptive")
    return out[:n.value], acc[:s.value], dr[:s.value]


def ls_generate_full(h, prompt, max_new):
    a, p = _i32(prompt)
    out = np.zeros(max_new, np.int32)
    n = C.c_int32()
    _ck(lib().ls_generate_full(h, p, a.size, max_new, out.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(n)),
        "ls_generate_full")
    return out[:n.value]


def ls_generate_early(h, prompt, exit_layer, max_new):
    a, p = _i32(prompt)
    out = np.zeros(max_new, np.int32)
    n = C.c_int32()
    _ck(lib().ls_generate_early(h, p, a.size, exit_layer, max_new, out.ctypes.data_as(C.POINTER(C.c_int32)),
                                C.byref(n)), "ls_generate_early")
    return out[:n.value]


def ls_prefill(h, prompt, layers=0):
    a, p = _i32(prompt)
    _ck(lib().ls_prefill(h, p, a.size, layers), "ls_prefill")


def ls_decode(h, exit_layer, num_draft, max_new):
    _ck(lib().ls_decode(h, exit_layer, num_draft, max_new), "ls_decode")


LS_DECODE_NO_EXIT_CACHE = 1


def ls_decode_flags(h, exit_layer, num_draft, max_new, flags):
    _ck(lib().ls_decode_flags(h, exit_layer, num_draft, max_new, flags), "ls_decode_flags")


def ls_decode_adaptive(h, exit_layer, max_draft, min_margin, max_new):
    _ck(lib().ls_decode_adaptive(h, exit_layer, max_draft, float(min_margin), max_new), "ls_decode_adaptive")


def ls_read_drafted(h, max_new):
    dr = np.zeros(max_new, np.int32)
    s = C.c_int32()
    _ck(lib().ls_read_drafted(h, dr.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(s)), "ls_read_drafted")
    return dr[:s.value]


def ls_read_output(h, max_new):
    out, acc = np.zeros(max_new, np.int32), np.zeros(max_new, np.int32)
    n, s = C.c_int32(), C.c_int32()
    _ck(lib().ls_read_output(h, out.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(n),
                             acc.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(s)), "ls_read_output")
    return out[:n.value], acc[:s.value]


def _cat_prompts(prompts):
    lens = np.asarray([len(p) for p in prompts], dtype=np.int32)
    flat = np.ascontiguousarray(np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts]))
    return flat, lens


def ls_prefill_batch(h, prompts):
    flat, lens = _cat_prompts(prompts)
    ipt = C.POINTER(C.c_int32)
    _ck(lib().ls_prefill_batch(h, len(prompts), flat.ctypes.data_as(ipt), lens.ctypes.data_as(ipt)), "ls_prefill_batch")


def ls_decode_batch(h, exit_layer, num_draft, max_new):
    _ck(lib().ls_decode_batch(h, exit_layer, num_draft, max_new), "ls_decode_batch")


def ls_read_output_seq(h, seq, max_new):
    out, acc = np.zeros(max_new, np.int32), np.zeros(max_new, np.int32)
    n, s = C.c_int32(), C.c_int32()
    ipt = C.POINTER(C.c_int32)
    _ck(lib().ls_read_output_seq(h, seq, out.ctypes.data_as(ipt), C.byref(n), acc.ctypes.data_as(ipt), C.byref(s)),
        "ls_read_output_seq")
    return out[:n.value], acc[:s.value]


def ls_generate_batch(h, prompts, exit_layer, num_draft, max_new):
    """-> [(ids, accepted_per_step)] per sequence"""
    flat, lens = _cat_prompts(prompts)
    B = len(prompts)
    out, acc = np.zeros((B, max_new), np.int32), np.zeros((B, max_new), np.int32)
    n, st = np.zeros(B, np.int32), np.zeros(B, np.int32)
    ipt = C.POINTER(C.c_int32)
    _ck(lib().ls_generate_batch(h, B, flat.ctypes.data_as(ipt), lens.ctypes.data_as(ipt), exit_layer, num_draft, max_new,
                                out.ctypes.data_as(ipt), n.ctypes.data_as(ipt), acc.ctypes.data_as(ipt),
                                st.ctypes.data_as(ipt)), "ls_generate_batch")
    return [(out[b, :n[b]].copy(), acc[b, :st[b]].copy()) for b in range(B)]


def ls_debug_next_logits(h, vocab):
    """after ls_prefill: final logits of the last prompt token on top of the prompt pass's cache"""
    out = np.empty(vocab, np.float32)
    _ck(lib().ls_debug_next_logits(h, out.ctypes.data_as(C.POINTER(C.c_float))), "ls_debug_next_logits")
    return out


def ls_debug_logits(h, ids, exit_layer, vocab, want_exit=True, want_final=True):
    a, p = _i32(ids)
    ex = np.empty((a.size, vocab), np.float32) if want_exit else None
    fi = np.empty((a.size, vocab), np.float32) if want_final else None
    fp = C.POINTER(C.c_float)
    _ck(lib().ls_debug_logits(h, p, a.size, exit_layer, ex.ctypes.data_as(fp) if want_exit else None,
                              fi.ctypes.data_as(fp) if want_final else None), "ls_debug_logits")
    return ex, fi


def ls_get_stats(h) -> ls_stats:
    s = ls_stats()
    _ck(lib().ls_get_stats(h, C.byref(s)), "ls_get_stats")
    return s


# ------------------------------------------------------------------ single operations (torch CUDA tensors)
def ls_op_embed(emb, tok, x):
    M, D = x.shape
    _ck(lib().ls_op_embed(_dev(emb), _dev(tok), M, D, emb.shape[0], _dev(x), _stream()), "ls_op_embed")


def ls_op_rmsnorm(x, gain, eps, out):
    M, D = x.shape
    _ck(lib().ls_op_rmsnorm(_dev(x), _dev(gain), M, D, eps, _dev(out), _stream()), "ls_op_rmsnorm")


def ls_op_chain(on):
    _ck(lib().ls_op_chain(int(bool(on))), "ls_op_chain")


def ls_op_linear(path, w, h, out, residual=False):
    (N, K), M = w.shape, h.shape[0]
    _ck(lib().ls_op_linear(path, _dev(w), _dev(h), M, N, K, _dev(out), int(residual), _stream()), "ls_op_linear")


def ls_op_gate_up_swiglu(path, w_gate, w_up, h, out):
    (F, K), M = w_gate.shape, h.shape[0]
    _ck(lib().ls_op_gate_up_swiglu(path, _dev(w_gate), _dev(w_up), _dev(h), M, F, K, _dev(out), _stream()),
        "ls_op_gate_up_swiglu")


def ls_op_lm_head_scratch_bytes(V):
    return lib().ls_op_lm_head_scratch_bytes(V)


def ls_op_lm_head_argmax(path, w, h, scratch, tok, logits=None):
    (V, K), M = w.shape, h.shape[0]
    _ck(lib().ls_op_lm_head_argmax(path, _dev(w), _dev(h), M, V, K, _dev(scratch), _dev(tok), _dev(logits),
                                   _stream()), "ls_op_lm_head_argmax")


LS_OP_LM_HEAD_STATIC_MAX_VOCAB = 131072


def ls_op_lm_head_argmax_static(path, w, h, tok):
    """LM head + argmax for callers that have no scratch buffer to give (they cannot
    allocate): the candidates go to a buffer inside the library.  Vocabulary at most
    LS_OP_LM_HEAD_STATIC_MAX_VOCAB; calls must not overlap on the GPU."""
    (V, K), M = w.shape, h.shape[0]
    _ck(lib().ls_op_lm_head_argmax_static(path, _dev(w), _dev(h), M, V, K, _dev(tok), _stream()),
        "ls_op_lm_head_argmax_static")


def ls_op_rope_append(qkv, pos0, Hq, Hkv, hd, theta, page_size, page_table, max_seq, q_out, k_pages, v_pages):
    _ck(lib().ls_op_rope_append(_dev(qkv), qkv.shape[0], pos0, Hq, Hkv, hd, theta, page_size, _dev(page_table),
                                max_seq, _dev(q_out), _dev(k_pages), _dev(v_pages), _stream()), "ls_op_rope_append")


def ls_op_qkv_rope_append(path, wq, wk, wv, h, pos0, Hq, Hkv, hd, theta, page_size, page_table, max_seq, q_out,
                          k_pages, v_pages):
    M, K = h.shape
    _ck(lib().ls_op_qkv_rope_append(path, _dev(wq), _dev(wk), _dev(wv), _dev(h), M, K, pos0, Hq, Hkv, hd, theta,
                                    page_size, _dev(page_table), max_seq, _dev(q_out), _dev(k_pages), _dev(v_pages),
                                    _stream()), "ls_op_qkv_rope_append")


def ls_op_attention(q, pos0, Hq, Hkv, hd, page_size, page_table, max_seq, k_pages, v_pages, out):
    _ck(lib().ls_op_attention(_dev(q), q.shape[0], pos0, Hq, Hkv, hd, page_size, _dev(page_table), max_seq,
                              _dev(k_pages), _dev(v_pages), _dev(out), _stream()), "ls_op_attention")


def ls_op_gemm(a, b, c, accumulate=False, status=None):
    """c[M, N] (+)= a[M, K] @ b[N, K].T  (bf16 inputs, fp32 c, tcgen05 tensor cores)"""
    (M, K), N = a.shape, b.shape[0]
    _ck(lib().ls_op_gemm(_dev(a), _dev(b), M, N, K, _dev(c), c.stride(0), int(accumulate), _dev(status), _stream()),
        "ls_op_gemm")


def ls_op_prefill_attention(q, pos0, Hq, Hkv, hd, page_size, page_table, max_seq, k_pages, v_pages, out, status=None):
    _ck(lib().ls_op_prefill_attention(_dev(q), q.shape[0], pos0, Hq, Hkv, hd, page_size, _dev(page_table), max_seq,
                                      _dev(k_pages), _dev(v_pages), _dev(out), _dev(status), _stream()),
        "ls_op_prefill_attention")


# ---- 4-bit weights and the 4-bit cache
def _bad(what):
    raise LsError(LS_ERR_INVALID_ARG, what)


def _arg(t, dtype, dev, what):
    """device pointer of a contiguous CUDA tensor of the type the entry point reads, on device dev"""
    if t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    _bad(f"{what}: a contiguous {dtype} tensor is needed, on the CUDA device of the others")


def _status(t, dev):
    return None if t is None else _arg(t, _torch.i32, dev, "status")


def _stream_on(dev):
    """handle of the current stream, which has to be one of the operands' device"""
    if dev < 0 or dev != _torch.device():
        _bad("operands on the current CUDA device are needed")
    return _torch.stream(dev)


@functools.lru_cache(maxsize=4096)
def ls_op_w4_bytes(N, K, group):
    return lib().ls_op_w4_bytes(N, K, group)


def _packed(packed, N, K, group, dev):
    """device pointer of packed weights (uint8), which must be large enough for [N, K]"""
    if packed.numel() < ls_op_w4_bytes(N, K, group):
        raise LsError(LS_ERR_CAPACITY, "packed weights")
    return _arg(packed, _torch.u8, dev, "packed weights")


def ls_op_quantize_w4(w, group, packed):
    """bf16 [N, K] -> packed 4-bit weights (uint8, ls_op_w4_bytes(N, K, group) of them)"""
    (N, K), dev = w.shape, w.get_device()
    p = _packed(packed, N, K, group, dev)
    _ck(lib().ls_op_quantize_w4(_arg(w, _torch.bf16, dev, "w"), N, K, group, p, _stream_on(dev)), "ls_op_quantize_w4")


def ls_op_expand_w4(packed, group, out):
    (N, K), dev = out.shape, out.get_device()
    p = _packed(packed, N, K, group, dev)
    _ck(lib().ls_op_expand_w4(p, N, K, group, _arg(out, _torch.bf16, dev, "out"), _stream_on(dev)), "ls_op_expand_w4")


def ls_op_linear_w4(packed, group, h, out, residual=False):
    """out[M, N] (+)= h[M, K] @ W.T of the packed weights W [N, K]"""
    (M, K), (rows, N), dev = h.shape, out.shape, h.get_device()
    if rows != M:
        _bad("ls_op_linear_w4: rows of h and out")
    p = _packed(packed, N, K, group, dev)
    _ck(lib().ls_op_linear_w4(p, _arg(h, _torch.bf16, dev, "h"), M, N, K, group, _arg(out, _torch.f32, dev, "out"), int(residual), _stream_on(dev)),
        "ls_op_linear_w4")


def ls_op_kv4_page_bytes(Hkv, hd, page_size):
    return lib().ls_op_kv4_page_bytes(Hkv, hd, page_size)


def _pool(pages, Hkv, hd, page_size):
    """number of pages of a pool (uint8, whole pages)"""
    per, size = Hkv * page_size * (hd + hd // 8), pages.numel()  # ls_op_kv4_page_bytes, which checks more
    if per <= 0 or size % per:
        _bad("pages of a 4-bit cache")
    return size // per


def _rows(pos0, table, n_seq):
    """entries per sequence of a page table int32 [n_seq, entries]; pos0 int32 [n_seq]"""
    shape = table.shape
    if pos0.numel() != n_seq or len(shape) != 2 or shape[0] != n_seq:
        _bad("pos0 [n_seq] and page table [n_seq, entries]")
    return shape[1]


def ls_op_append_kv4(k, v, pos0, page_size, table, max_seq, pages, status=None):
    """k, v bf16 [n_seq, M, Hkv, hd], of any strides but equal ones (in dimensions of more than one), channels contiguous"""
    (n_seq, M, Hkv, hd), dev = k.shape, k.get_device()
    n_pages, entries = _pool(pages, Hkv, hd, page_size), _rows(pos0, table, n_seq)
    stride = k.stride()
    if v.shape != k.shape or stride[3] != 1 or dev < 0 or v.get_device() != dev or \
            k.dtype is not _torch.bf16 or v.dtype is not _torch.bf16 or \
            (v.stride() != stride and any(n > 1 and a != b for n, a, b in zip(k.shape, stride, v.stride()))):
        _bad("ls_op_append_kv4: k and v")
    _ck(lib().ls_op_append_kv4(k.data_ptr(), v.data_ptr(), stride[0], stride[1], stride[2], n_seq, M,
                               _arg(pos0, _torch.i32, dev, "pos0"), Hkv, hd, page_size, _arg(table, _torch.i32, dev, "page table"), entries, max_seq,
                               _arg(pages, _torch.u8, dev, "pages"), n_pages, _status(status, dev), _stream_on(dev)), "ls_op_append_kv4")


def ls_op_expand_kv4(pages, pos0, M, page_size, table, max_seq, out_table, k_pages, v_pages, status=None):
    """k_pages, v_pages bf16 [n_out_pages, Hkv, page_size, hd]"""
    (n_out, Hkv, ps, hd), dev = k_pages.shape, k_pages.get_device()
    n_seq = table.shape[0]
    n_pages, entries = _pool(pages, Hkv, hd, page_size), _rows(pos0, table, n_seq)
    if ps != page_size or v_pages.shape != k_pages.shape or out_table.shape != table.shape:
        _bad("ls_op_expand_kv4: k_pages, v_pages and their table")
    _ck(lib().ls_op_expand_kv4(_arg(pages, _torch.u8, dev, "pages"), n_pages, n_seq, M, _arg(pos0, _torch.i32, dev, "pos0"), Hkv, hd, page_size,
                               _arg(table, _torch.i32, dev, "page table"), entries, max_seq, _arg(out_table, _torch.i32, dev, "out page table"),
                               _arg(k_pages, _torch.bf16, dev, "k_pages"), _arg(v_pages, _torch.bf16, dev, "v_pages"), n_out,
                               _status(status, dev), _stream_on(dev)), "ls_op_expand_kv4")


@functools.lru_cache(maxsize=4096)
def ls_op_attention_kv4_scratch_bytes(n_seq, M, Hq, Hkv, hd, max_seq):
    return lib().ls_op_attention_kv4_scratch_bytes(n_seq, M, Hq, Hkv, hd, max_seq)


def ls_op_attention_kv4(q, pos0, Hkv, hd, page_size, table, max_seq, pages, out, status=None, scratch=None):
    """q, out bf16 [n_seq, M, Hq * hd].  scratch: uint8, ls_op_attention_kv4_scratch_bytes of them; None allocates them
    where the call can use any (torch's allocator hands them out and takes them back in stream order)."""
    (n_seq, M, width), dev = q.shape, q.get_device()
    n_pages, entries = _pool(pages, Hkv, hd, page_size), _rows(pos0, table, n_seq)
    if width % hd or out.shape != q.shape:
        _bad("ls_op_attention_kv4: q and out")
    Hq = width // hd
    need = ls_op_attention_kv4_scratch_bytes(n_seq, M, Hq, Hkv, hd, max_seq)
    if scratch is None and need:
        scratch = _torch.empty(need, dtype=_torch.u8, device=q.device)
    elif scratch is not None and scratch.numel() < need:
        raise LsError(LS_ERR_CAPACITY, "ls_op_attention_kv4: scratch")
    _ck(lib().ls_op_attention_kv4(_arg(q, _torch.bf16, dev, "q"), n_seq, M, _arg(pos0, _torch.i32, dev, "pos0"), Hq, Hkv, hd, page_size,
                                  _arg(table, _torch.i32, dev, "page table"), entries, max_seq, _arg(pages, _torch.u8, dev, "pages"), n_pages,
                                  _arg(out, _torch.bf16, dev, "out"), None if scratch is None else _arg(scratch, _torch.u8, dev, "scratch"), _status(status, dev),
                                  _stream_on(dev)), "ls_op_attention_kv4")


# ---- 8-bit values with a scale for each block of 128
LS_BF16, LS_F32 = 0, 1
LS_F8_MAX_ROWS = 1 << 22


@functools.lru_cache(maxsize=4096)
def ls_op_f8_scale_bytes(M, K, block_rows=1):
    if not (0 < M <= LS_F8_MAX_ROWS and 0 < K <= 1 << 28 and block_rows in (1, 128)):  # 32 bits of them go to the library
        return 0
    return lib().ls_op_f8_scale_bytes(M, K, block_rows)


def _held(codes, scales, M, K, block_rows, dev, what):
    """device pointers of codes float8_e4m3fn [M, K] and their scales (uint8, ls_op_f8_scale_bytes of them)"""
    if codes.dtype is not _torch.f8 or scales.dtype is not _torch.u8 or codes.get_device() != dev or scales.get_device() != dev or \
            not codes.is_contiguous() or not scales.is_contiguous():
        _bad(f"{what}: contiguous codes (float8_e4m3fn) and scales (uint8) are needed, on the CUDA device of the others")
    need = ls_op_f8_scale_bytes(M, K, block_rows)
    if not need:
        _bad(f"{what}: a shape of the format is needed, in blocks of 1 or 128 rows")
    if scales.numel() < need:
        raise LsError(LS_ERR_CAPACITY, f"{what}: scales")
    return codes.data_ptr(), scales.data_ptr()


def _strided(t, shape, dev, what):
    """(device pointer, type, row stride) of a bf16 or fp32 tensor of some shape [M, K] with contiguous columns"""
    dtype, stride = t.dtype, t.stride()
    kind = LS_F32 if dtype is _torch.f32 else LS_BF16 if dtype is _torch.bf16 else -1
    if kind < 0 or t.shape != shape or t.get_device() != dev or (stride[1] != 1 and shape[1] > 1):
        _bad(f"{what}: a bf16 or fp32 tensor {tuple(shape)} with contiguous columns is needed, on the CUDA device of the others")
    return t.data_ptr(), kind, stride[0]


def ls_op_quantize_f8(x, codes, scales, block_rows=1):
    """x [M, K], bf16 or fp32 -> codes (float8_e4m3fn [M, K]) and scales (uint8), of one row's or 128 rows' blocks of 128 columns"""
    shape, dev = codes.shape, codes.get_device()
    M, K = shape
    c, s = _held(codes, scales, M, K, block_rows, dev, "ls_op_quantize_f8")
    xp, kind, ld = _strided(x, shape, dev, "x")
    rc = lib().ls_op_quantize_f8(xp, kind, ld, M, K, block_rows, c, s, _stream_on(dev))
    if rc:
        raise LsError(rc, "ls_op_quantize_f8")


def ls_op_expand_f8(codes, scales, out, block_rows=1):
    """codes and scales -> bf16 [M, K]"""
    shape, dev = codes.shape, codes.get_device()
    M, K = shape
    c, s = _held(codes, scales, M, K, block_rows, dev, "ls_op_expand_f8")
    if out.shape != shape:
        _bad("ls_op_expand_f8: out")
    rc = lib().ls_op_expand_f8(c, s, M, K, block_rows, _arg(out, _torch.bf16, dev, "out"), _stream_on(dev))
    if rc:
        raise LsError(rc, "ls_op_expand_f8")


def ls_op_rmsnorm_f8(x, gain, eps, codes, scales, delta=None, x_out=None):
    """codes and scales of the RMSNorm of x + delta [M, D], which goes to x_out (may be x) if it is given"""
    shape, dev = codes.shape, codes.get_device()
    M, D = shape
    c, s = _held(codes, scales, M, D, 1, dev, "ls_op_rmsnorm_f8")
    xp, kind, ldx = _strided(x, shape, dev, "x")
    dp, dkind, ldd = (None, LS_F32, 0) if delta is None else _strided(delta, shape, dev, "delta")
    op, okind, ldo = (xp, kind, ldx) if x_out is x else (None, kind, 0) if x_out is None else _strided(x_out, shape, dev, "x_out")
    if okind != kind or gain.numel() != D:
        _bad("ls_op_rmsnorm_f8: x_out of x's type, gain [D]")
    rc = lib().ls_op_rmsnorm_f8(xp, kind, ldx, dp, dkind, ldd, op, ldo, _arg(gain, _torch.bf16, dev, "gain"), M, D, eps, c, s, _stream_on(dev))
    if rc:
        raise LsError(rc, "ls_op_rmsnorm_f8")


def ls_op_swiglu_f8(gate, up, codes, scales):
    """codes and scales of silu(gate) * up [M, F]; gate and up of one type and row stride"""
    shape, dev = codes.shape, codes.get_device()
    M, F = shape
    c, s = _held(codes, scales, M, F, 1, dev, "ls_op_swiglu_f8")
    gp, kind, ld = _strided(gate, shape, dev, "gate")
    upp, ukind, uld = _strided(up, shape, dev, "up")
    if kind != ukind or (ld != uld and M > 1):
        _bad("ls_op_swiglu_f8: gate and up of one type and row stride")
    rc = lib().ls_op_swiglu_f8(gp, upp, kind, ld, M, F, c, s, _stream_on(dev))
    if rc:
        raise LsError(rc, "ls_op_swiglu_f8")


def ls_op_linear_f8(w_codes, w_scales, h_codes, h_scales, out, add=None, status=None):
    """out[M, N] = (add +) h @ W.T of weights [N, K] in blocks of 128 x 128 and tokens [M, K] in blocks of 1 x 128; out bf16
    or fp32, add of its type (may be out)"""
    (N, K), (M, Kh), dev = w_codes.shape, h_codes.shape, h_codes.get_device()
    if K != Kh:
        _bad("ls_op_linear_f8: columns of w and h")
    wc, ws = _held(w_codes, w_scales, N, K, 128, dev, "ls_op_linear_f8: w")
    hc, hs = _held(h_codes, h_scales, M, K, 1, dev, "ls_op_linear_f8: h")
    op, kind, ldo = _strided(out, (M, N), dev, "out")
    ap, akind, lda = (None, kind, 0) if add is None else (op, kind, ldo) if add is out else _strided(add, (M, N), dev, "add")
    if akind != kind:
        _bad("ls_op_linear_f8: add of out's type")
    rc = lib().ls_op_linear_f8(wc, ws, hc, hs, M, N, K, op, kind, ldo, ap, lda, None if status is None else _status(status, dev), _stream_on(dev))
    if rc:
        raise LsError(rc, "ls_op_linear_f8")


def ls_op_accept(draft, verified, d, state, out_ids, accepted):
    _ck(lib().ls_op_accept(_dev(draft), _dev(verified), d, _dev(state), _dev(out_ids), _dev(accepted), _stream()),
        "ls_op_accept")


# ------------------------------------------------------------------ convenience: own the device memory of one model
class Model:
    """Allocates the workspace with torch, creates the handle, keeps everything alive."""

    def __init__(self, shape, weights: dict, max_seq: int, page_size: int = 64, max_draft: int = 8,
                 eos_id: int = -1, linear_path: int = LS_LINEAR_AUTO):
        import torch
        self.shape = shape
        self.cfg = make_config(shape, max_seq, page_size, max_draft, eos_id, linear_path)
        nbytes = ls_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise LsError(LS_ERR_INVALID_ARG, "ls_workspace_bytes")
        self.weights = weights
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        self.h = ls_model_create(self.cfg, weights, self.workspace)

    def close(self):
        if getattr(self, "h", None):
            ls_model_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def generate(self, prompt, exit_layer, num_draft, max_new):
        return ls_generate(self.h, prompt, exit_layer, num_draft, max_new)

    def generate_adaptive(self, prompt, exit_layer, max_draft, min_margin, max_new):
        return ls_generate_adaptive(self.h, prompt, exit_layer, max_draft, min_margin, max_new)

    def generate_full(self, prompt, max_new):
        return ls_generate_full(self.h, prompt, max_new)

    def generate_early(self, prompt, exit_layer, max_new):
        return ls_generate_early(self.h, prompt, exit_layer, max_new)

    def generate_batch(self, prompts, exit_layer, num_draft, max_new):
        return ls_generate_batch(self.h, prompts, exit_layer, num_draft, max_new)

    def debug_logits(self, ids, exit_layer, want_exit=True, want_final=True):
        return ls_debug_logits(self.h, ids, exit_layer, self.shape.vocab, want_exit, want_final)

    def stats(self):
        return ls_get_stats(self.h)
