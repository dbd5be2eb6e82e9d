"""Python binding of ``libdels.so``, the DeLS-Spec drafting hot path on GB300.

Argument marshalling only: every step of the drafting loop, the combine and
the verification runs in the library's CUDA kernels. Functions named
``dels_*`` mirror the C ABI in ``include/dels.h`` one to one and take torch
tensors (or raw integer device pointers) in place of the C pointers. The
``Drafter`` helper keeps a local head's weight pointers and a workspace for
repeated calls. There is no CPU fallback: if ``libdels.so`` has not been
built, every call raises ``RuntimeError``.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Dict, Optional

import torch

__all__ = [
    "DELS_OK", "DELS_F32", "DELS_BF16",
    "DELS_HEAD_GRU", "DELS_HEAD_MLP", "DELS_HEAD_XFMR", "DELS_HEAD_MARKOV",
    "DELS_STATUS_NONFINITE", "DELS_STATUS_TIMEOUT", "DELS_STATUS_BAD_TOKEN",
    "DELS_ERR_NULL_POINTER", "DELS_ERR_BAD_SHAPE", "DELS_ERR_BAD_DTYPE", "DELS_ERR_ALIGNMENT",
    "DELS_ERR_WORKSPACE", "DELS_ERR_UNSUPPORTED", "DELS_ERR_CUDA", "DELS_ERR_TOO_LARGE",
    "DelsError", "LocalHead", "lib", "library_path", "exported_symbols",
    "dels_draft_workspace_bytes", "dels_draft_block", "dels_draft_block_weighted",
    "dels_draft_state_bytes", "dels_draft_block_sampled",
    "dels_verify_sampled_workspace_bytes", "dels_verify_block_sampled",
    "dels_combine_workspace_bytes", "dels_combine_argmax", "dels_combine_argmax_noalloc",
    "dels_verify_workspace_bytes", "dels_verify_block",
    "dels_read_status", "dels_prior_from_counts", "dels_status_string", "dels_version",
    "dels_profile_enable", "dels_profile_reset", "dels_profile_read", "KCLASS",
    "dels_gru_input_table_bytes", "dels_gru_build_input_table", "gru_input_table",
    "dels_selftest_timeout_bytes", "dels_selftest_timeout", "dels_selftest_gumbel",
    "dels_prior_workspace_bytes", "dels_prior_count", "dels_prior_log", "dels_prior_estimate", "estimate_prior",
    "make_head", "Drafter", "dtype_code",
    "Rows", "Teacher", "dels_score_workspace_bytes", "dels_score_rows",
    "dels_distill_state_bytes", "dels_distill_workspace_bytes", "dels_distill_loss", "dels_distill_grad",
    "dels_distill_step", "rows_of", "teacher_of", "TokenScorer", "Distiller", "distill_loss",
]

DELS_OK = 0
DELS_F32, DELS_BF16 = 0, 1
DELS_HEAD_GRU, DELS_HEAD_MLP, DELS_HEAD_XFMR, DELS_HEAD_MARKOV = 0, 1, 2, 3
DELS_STATUS_NONFINITE, DELS_STATUS_TIMEOUT, DELS_STATUS_BAD_TOKEN = 1, 2, 4
(DELS_ERR_NULL_POINTER, DELS_ERR_BAD_SHAPE, DELS_ERR_BAD_DTYPE, DELS_ERR_ALIGNMENT, DELS_ERR_WORKSPACE,
 DELS_ERR_UNSUPPORTED, DELS_ERR_CUDA, DELS_ERR_TOO_LARGE) = -1, -2, -3, -4, -5, -6, -7, -8

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libdels.so")
_lib = None

# name -> (restype, argtypes); the C ABI of include/dels.h
_vp, _i, _f, _d, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_double, ctypes.c_size_t


class LocalHead(ctypes.Structure):
    """Mirror of ``dels_local_head``."""

    _fields_ = [
        ("kind", ctypes.c_int), ("wdtype", ctypes.c_int),
        ("d_model", ctypes.c_int), ("d_hidden", ctypes.c_int), ("d_rank", ctypes.c_int),
        ("window", ctypes.c_int), ("n_layers", ctypes.c_int), ("n_heads", ctypes.c_int),
        ("max_pos", ctypes.c_int),
        ("emb", ctypes.c_void_p), ("w", ctypes.c_void_p * 8), ("w_vocab", ctypes.c_void_p),
    ]


class Rows(ctypes.Structure):
    """Mirror of ``dels_rows``."""

    _fields_ = [
        ("long_logits", ctypes.c_void_p), ("short_logits", ctypes.c_void_p), ("dtype", ctypes.c_int),
        ("long_stride", ctypes.c_longlong), ("short_stride", ctypes.c_longlong),
        ("log_prior", ctypes.c_void_p), ("alpha", ctypes.c_void_p), ("beta", ctypes.c_void_p),
        ("n_weights", ctypes.c_int), ("temperature", ctypes.c_float),
    ]


class Teacher(ctypes.Structure):
    """Mirror of ``dels_teacher``."""

    _fields_ = [
        ("ids", ctypes.c_void_p), ("logprob", ctypes.c_void_p), ("k", ctypes.c_int), ("tail", ctypes.c_int),
        ("row_weight", ctypes.c_void_p),
    ]


_ROWS, _TEACHER, _ll = ctypes.POINTER(Rows), ctypes.POINTER(Teacher), ctypes.c_longlong

_SIGS = {
    "dels_selftest_timeout_bytes": (_sz, []),
    "dels_selftest_timeout": (_i, [_vp, _sz, _vp]),
    "dels_selftest_gumbel": (_i, [_vp, _vp, ctypes.c_longlong, _vp]),
    "dels_gru_input_table_bytes": (_sz, [ctypes.POINTER(LocalHead), _i]),
    "dels_gru_build_input_table": (_i, [ctypes.POINTER(LocalHead), _i, _vp, _sz, _vp, _sz, _vp]),
    "dels_draft_workspace_bytes": (_sz, [ctypes.POINTER(LocalHead), _i, _i, _i]),
    "dels_draft_block": (_i, [ctypes.POINTER(LocalHead), _vp, _i, _vp, _f, _f, _i, _i, _i, _vp, _vp, _vp, _vp, _sz,
                              _vp]),
    "dels_draft_block_weighted": (_i, [ctypes.POINTER(LocalHead), _vp, _i, _vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp,
                                       _vp, _sz, _vp]),
    "dels_draft_state_bytes": (_sz, [ctypes.POINTER(LocalHead), _i, _i]),
    "dels_draft_block_sampled": (_i, [ctypes.POINTER(LocalHead), _vp, _i, _vp, _vp, _vp, _i, _i, _i, ctypes.c_uint64,
                                      ctypes.c_uint64, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "dels_verify_sampled_workspace_bytes": (_sz, [ctypes.POINTER(LocalHead), _i, _i, _i, _i]),
    "dels_verify_block_sampled": (_i, [ctypes.POINTER(LocalHead), _vp, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _i, _i,
                                       _i, _i, ctypes.c_uint64, ctypes.c_uint64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dels_combine_workspace_bytes": (_sz, [_i, _i, _i]),
    "dels_combine_argmax": (_i, [_vp, _vp, _i, _vp, _f, _f, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dels_combine_argmax_noalloc": (_i, [_vp, _vp, _i, _vp, _f, _f, _i, _i, _vp, _vp, _vp, _vp]),
    "dels_verify_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "dels_verify_block": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dels_read_status": (_i, [_vp, _vp, ctypes.POINTER(ctypes.c_int32)]),
    "dels_prior_from_counts": (_i, [_vp, _i, _d, _vp]),
    "dels_prior_workspace_bytes": (_sz, [_i, ctypes.c_int64]),
    "dels_prior_count": (_i, [_vp, _vp, ctypes.c_int64, _i, _vp, _vp, _vp, _sz, _vp]),
    "dels_prior_log": (_i, [_vp, _i, _d, _vp, _vp, _sz, _vp]),
    "dels_prior_estimate": (_i, [_vp, _vp, ctypes.c_int64, _i, _d, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dels_score_workspace_bytes": (_sz, [_i, _i]),
    "dels_score_rows": (_i, [_ROWS, _i, _i, _vp, _i, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dels_distill_state_bytes": (_sz, [_i]),
    "dels_distill_workspace_bytes": (_sz, [_i, _i]),
    "dels_distill_loss": (_i, [_ROWS, _i, _i, _TEACHER, _vp, _vp, _sz, _vp, _sz, _vp]),
    "dels_distill_grad": (_i, [_ROWS, _i, _i, _TEACHER, _vp, _vp, _sz, _vp, _ll, _vp, _vp, _vp]),
    "dels_distill_step": (_i, [_ROWS, _i, _i, _TEACHER, _vp, _vp, _ll, _vp, _vp, _vp, _sz, _vp]),
    "dels_status_string": (ctypes.c_char_p, [_i]),
    "dels_version": (_i, []),
    "dels_profile_enable": (_i, [_i]),
    "dels_profile_reset": (_i, []),
    "dels_profile_read": (_i, [_i, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_double)]),
}

# kernel classes of the optional profiler
KCLASS = {"vocab_combine": 0, "head_gemm": 1, "head_misc": 2, "merge": 3, "pos0": 4, "verify": 5, "combine": 6,
          "draft_block": 7, "prior": 8, "score": 9, "distill": 10}


def exported_symbols():
    """Names of the C ABI entry points this binding expects the library to export."""
    return list(_SIGS)


class DelsError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {dels_status_string(code)} ({code})")


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded ``libdels.so`` (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} not found: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


# ----------------------------------------------------------------------------- marshalling helpers

def _ptr(x) -> Optional[int]:
    """Device address of a CUDA tensor, or an integer address passed through.

    Every pointer the library's entry points take through this helper is a
    device pointer into a row-major layout, so a host tensor or a strided
    view is refused here instead of reaching a kernel."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        if not x.is_cuda:
            raise ValueError("expected a CUDA tensor: the library's entry points take device pointers")
        if not x.is_contiguous():
            raise ValueError("expected a contiguous tensor: the library's layouts are dense row-major")
        return x.data_ptr()
    return int(x)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if torch.cuda.is_initialized():       # the current device's current stream, without the object around it
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def dtype_code(t) -> int:
    if isinstance(t, torch.Tensor):
        t = t.dtype
    if t == torch.float32:
        return DELS_F32
    if t == torch.bfloat16:
        return DELS_BF16
    raise ValueError(f"unsupported dtype {t}")


def _check(code: int, where: str):
    if code != DELS_OK:
        raise DelsError(code, where)


# ----------------------------------------------------------------------------- the C ABI, by name

def dels_version() -> int:
    return lib().dels_version()


def dels_status_string(code: int) -> str:
    return lib().dels_status_string(int(code)).decode()


def dels_selftest_timeout_bytes() -> int:
    return lib().dels_selftest_timeout_bytes()


def dels_selftest_timeout(workspace, workspace_bytes: int, stream=None) -> int:
    return lib().dels_selftest_timeout(_ptr(workspace), workspace_bytes, _stream(stream))


def dels_selftest_gumbel(bits, g, n: int, stream=None) -> int:
    return lib().dels_selftest_gumbel(_ptr(bits), _ptr(g), n, _stream(stream))


def dels_gru_input_table_bytes(head: LocalHead, V: int) -> int:
    return lib().dels_gru_input_table_bytes(ctypes.byref(head), V)


def dels_gru_build_input_table(head: LocalHead, V: int, table, table_bytes: int, workspace, workspace_bytes: int,
                               stream=None) -> int:
    return lib().dels_gru_build_input_table(ctypes.byref(head), V, _ptr(table), table_bytes, _ptr(workspace),
                                            workspace_bytes, _stream(stream))


def gru_input_table(spec, weights: Dict[str, torch.Tensor], V: int, stream=None) -> torch.Tensor:
    """The GRU input table G = E W_ih^T [V, 3*d_hidden] float32 of a bf16 GRU
    head, built on the weights' device. Put it in the weights dict as
    ``input_table`` to have dels_draft_block read it."""
    head = make_head(spec, {k: v for k, v in weights.items() if k != "input_table"})
    nbytes = dels_gru_input_table_bytes(head, V)
    if nbytes == 0:
        raise DelsError(-6, "dels_gru_input_table_bytes")
    dev = weights["emb"].device
    table = torch.empty(nbytes // 4, dtype=torch.float32, device=dev).view(V, -1)
    ws = torch.zeros(256, dtype=torch.uint8, device=dev)
    _check(dels_gru_build_input_table(head, V, table, nbytes, ws, 256, stream), "dels_gru_build_input_table")
    st = dels_read_status(ws, stream)
    if st != 0:
        raise DelsError(st, "dels_gru_build_input_table (device status)")
    return table


def dels_draft_workspace_bytes(head: LocalHead, B: int, n: int, V: int) -> int:
    return lib().dels_draft_workspace_bytes(ctypes.byref(head), B, n, V)


def dels_draft_block(head: LocalHead, long_logits, logit_dtype: int, log_prior, alpha: float, beta: float,
                     B: int, n: int, V: int, out_tokens, out_logprob, out_top2_gap, workspace,
                     workspace_bytes: int, stream=None) -> int:
    r = lib().dels_draft_block(ctypes.byref(head), _ptr(long_logits), logit_dtype, _ptr(log_prior), alpha, beta,
                               B, n, V, _ptr(out_tokens), _ptr(out_logprob), _ptr(out_top2_gap),
                               _ptr(workspace), workspace_bytes, _stream(stream))
    return r


def dels_draft_block_weighted(head: LocalHead, long_logits, logit_dtype: int, log_prior, alpha, beta, B: int,
                              n: int, V: int, out_tokens, out_logprob, out_top2_gap, workspace,
                              workspace_bytes: int, stream=None) -> int:
    """Per-position fusion weights: ``alpha``/``beta`` are sequences of n floats
    (host; entry 0 unused)."""
    a = (ctypes.c_float * n)(*[float(x) for x in alpha])
    b = (ctypes.c_float * n)(*[float(x) for x in beta])
    return lib().dels_draft_block_weighted(ctypes.byref(head), _ptr(long_logits), logit_dtype, _ptr(log_prior),
                                           ctypes.cast(a, ctypes.c_void_p), ctypes.cast(b, ctypes.c_void_p), B, n, V,
                                           _ptr(out_tokens), _ptr(out_logprob), _ptr(out_top2_gap),
                                           _ptr(workspace), workspace_bytes, _stream(stream))


def _host_floats(xs, n):
    xs = [float(x) for x in xs]
    if len(xs) != n:
        raise ValueError(f"expected {n} per-position weights")
    arr = (ctypes.c_float * n)(*xs)
    return arr, ctypes.cast(arr, ctypes.c_void_p)


def dels_draft_state_bytes(head: LocalHead, B: int, n: int) -> int:
    return lib().dels_draft_state_bytes(ctypes.byref(head), B, n)


def dels_draft_block_sampled(head: LocalHead, long_logits, logit_dtype: int, log_prior, alpha, beta, B: int, n: int,
                             V: int, seed: int, step: int, out_tokens, out_logprob, out_key_gap, draft_state,
                             state_bytes: int, workspace, workspace_bytes: int, stream=None) -> int:
    """Temperature-1 drafting; ``alpha``/``beta`` are sequences of n floats (host)."""
    a, ap = _host_floats(alpha, n)
    b, bp = _host_floats(beta, n)
    return lib().dels_draft_block_sampled(ctypes.byref(head), _ptr(long_logits), logit_dtype, _ptr(log_prior), ap, bp,
                                          B, n, V, int(seed), int(step), _ptr(out_tokens), _ptr(out_logprob),
                                          _ptr(out_key_gap), _ptr(draft_state), state_bytes, _ptr(workspace),
                                          workspace_bytes, _stream(stream))


def dels_verify_sampled_workspace_bytes(head: LocalHead, B: int, n: int, V: int, target_dtype: int) -> int:
    return lib().dels_verify_sampled_workspace_bytes(ctypes.byref(head), B, n, V, target_dtype)


def dels_verify_block_sampled(head: LocalHead, draft_tokens, draft_logprob, draft_state, long_logits,
                              logit_dtype: int, log_prior, alpha, beta, target_logits, target_dtype: int, B: int,
                              n: int, V: int, seed: int, step: int, out_accept_len, out_bonus, out_bonus_gap,
                              workspace, workspace_bytes: int, stream=None) -> int:
    """Speculative-sampling verification of a temperature-1 block; ``alpha``/``beta`` host sequences of n."""
    a, ap = _host_floats(alpha, n)
    b, bp = _host_floats(beta, n)
    return lib().dels_verify_block_sampled(ctypes.byref(head), _ptr(draft_tokens), _ptr(draft_logprob),
                                           _ptr(draft_state), _ptr(long_logits), logit_dtype, _ptr(log_prior), ap, bp,
                                           _ptr(target_logits), target_dtype, B, n, V, int(seed), int(step),
                                           _ptr(out_accept_len), _ptr(out_bonus), _ptr(out_bonus_gap),
                                           _ptr(workspace), workspace_bytes, _stream(stream))


def dels_combine_workspace_bytes(rows: int, V: int, dtype: int) -> int:
    return lib().dels_combine_workspace_bytes(rows, V, dtype)


def dels_combine_argmax(long_logits, short_logits, dtype: int, log_prior, alpha: float, beta: float, rows: int,
                        V: int, out_token, out_logprob, out_top2_gap, workspace, workspace_bytes: int,
                        stream=None) -> int:
    return lib().dels_combine_argmax(_ptr(long_logits), _ptr(short_logits), dtype, _ptr(log_prior), alpha, beta,
                                     rows, V, _ptr(out_token), _ptr(out_logprob), _ptr(out_top2_gap),
                                     _ptr(workspace), workspace_bytes, _stream(stream))


def dels_combine_argmax_noalloc(long_logits, short_logits, dtype: int, log_prior, alpha: float, beta: float,
                                rows: int, V: int, out_token, out_logprob, out_top2_gap, stream=None) -> int:
    """dels_combine_argmax without a workspace: uses the library's fixed 4 MiB
    device scratch (for callers that cannot allocate device memory)."""
    return lib().dels_combine_argmax_noalloc(_ptr(long_logits), _ptr(short_logits), dtype, _ptr(log_prior), alpha,
                                             beta, rows, V, _ptr(out_token), _ptr(out_logprob), _ptr(out_top2_gap),
                                             _stream(stream))


def dels_verify_workspace_bytes(B: int, n: int, V: int, dtype: int) -> int:
    return lib().dels_verify_workspace_bytes(B, n, V, dtype)


def dels_verify_block(draft_tokens, target_logits, dtype: int, B: int, n: int, V: int, out_accept_len, out_bonus,
                      out_target_argmax, workspace, workspace_bytes: int, stream=None) -> int:
    return lib().dels_verify_block(_ptr(draft_tokens), _ptr(target_logits), dtype, B, n, V, _ptr(out_accept_len),
                                   _ptr(out_bonus), _ptr(out_target_argmax), _ptr(workspace), workspace_bytes,
                                   _stream(stream))


def dels_read_status(workspace, stream=None) -> int:
    out = ctypes.c_int32(0)
    _check(lib().dels_read_status(_ptr(workspace), _stream(stream), ctypes.byref(out)), "dels_read_status")
    return out.value


def dels_prior_from_counts(counts: torch.Tensor, lam: float = 1.0) -> torch.Tensor:
    """Host helper: float32 log prior [V] from int64 counts [V] (both CPU tensors)."""
    c = counts.detach().to("cpu", torch.int64).contiguous()
    out = torch.empty(c.numel(), dtype=torch.float32)
    _check(lib().dels_prior_from_counts(c.data_ptr(), c.numel(), float(lam), out.data_ptr()),
           "dels_prior_from_counts")
    return out


def dels_prior_workspace_bytes(V: int, N: int) -> int:
    return lib().dels_prior_workspace_bytes(V, N)


def dels_prior_count(tokens, loss_mask, N: int, V: int, counts, tally, workspace, workspace_bytes: int,
                     stream=None) -> int:
    """counts/tally: int64 (uint64 bit pattern) device tensors, accumulated."""
    return lib().dels_prior_count(_ptr(tokens), _ptr(loss_mask), N, V, _ptr(counts), _ptr(tally), _ptr(workspace),
                                  workspace_bytes, _stream(stream))


def dels_prior_log(counts, V: int, lam: float, out_log_prior, workspace, workspace_bytes: int, stream=None) -> int:
    return lib().dels_prior_log(_ptr(counts), V, float(lam), _ptr(out_log_prior), _ptr(workspace), workspace_bytes,
                                _stream(stream))


def dels_prior_estimate(tokens, loss_mask, N: int, V: int, lam: float, out_log_prior, out_counts, out_tally,
                        workspace, workspace_bytes: int, stream=None) -> int:
    return lib().dels_prior_estimate(_ptr(tokens), _ptr(loss_mask), N, V, float(lam), _ptr(out_log_prior),
                                     _ptr(out_counts), _ptr(out_tally), _ptr(workspace), workspace_bytes,
                                     _stream(stream))


def estimate_prior(tokens: torch.Tensor, loss_mask: torch.Tensor, V: int, lam: float = 1.0, stream=None):
    """Device unigram prior of a corpus: (log prior float32 [V], counts int64 [V],
    tally int64 [2] = positions counted, loss-masked ids outside [0, V))."""
    if tokens.dtype != torch.int32 or loss_mask.dtype not in (torch.uint8, torch.bool):
        raise ValueError("tokens must be int32 and loss_mask uint8")
    if tokens.numel() != loss_mask.numel():
        raise ValueError("tokens and loss_mask must have the same length")
    if not (tokens.is_contiguous() and loss_mask.is_contiguous()):
        raise ValueError("tokens and loss_mask must be contiguous")
    dev = tokens.device
    nbytes = dels_prior_workspace_bytes(V, tokens.numel())
    if nbytes == 0:
        raise DelsError(-2, "dels_prior_workspace_bytes")
    ws = torch.zeros(nbytes, dtype=torch.uint8, device=dev)
    out = torch.empty(V, dtype=torch.float32, device=dev)
    counts = torch.empty(V, dtype=torch.int64, device=dev)
    tally = torch.empty(2, dtype=torch.int64, device=dev)
    _check(dels_prior_estimate(tokens, loss_mask.view(torch.uint8), tokens.numel(), V, lam, out, counts, tally, ws,
                               nbytes, stream), "dels_prior_estimate")
    return out, counts, tally


def dels_score_workspace_bytes(rows: int, V: int) -> int:
    return lib().dels_score_workspace_bytes(rows, V)


def dels_score_rows(x: Rows, rows: int, V: int, tokens, top_k: int, out_logprob, out_entropy, out_top_ids,
                    out_top_logprob, workspace, workspace_bytes: int, stream=None) -> int:
    r = lib().dels_score_rows(ctypes.byref(x), rows, V, _ptr(tokens), top_k, _ptr(out_logprob), _ptr(out_entropy),
                              _ptr(out_top_ids), _ptr(out_top_logprob), _ptr(workspace), workspace_bytes,
                              _stream(stream))
    if r == DELS_OK:
        _written(out_logprob, out_entropy, out_top_ids, out_top_logprob)
    return r


def dels_distill_state_bytes(rows: int) -> int:
    return lib().dels_distill_state_bytes(rows)


def dels_distill_workspace_bytes(rows: int, V: int) -> int:
    return lib().dels_distill_workspace_bytes(rows, V)


def dels_distill_loss(x: Rows, rows: int, V: int, teacher: Teacher, out_loss, state, state_bytes: int, workspace,
                      workspace_bytes: int, stream=None) -> int:
    r = lib().dels_distill_loss(ctypes.byref(x), rows, V, ctypes.byref(teacher), _ptr(out_loss), _ptr(state),
                                state_bytes, _ptr(workspace), workspace_bytes, _stream(stream))
    if r == DELS_OK:
        _written(out_loss, state)
    return r


def dels_distill_grad(x: Rows, rows: int, V: int, teacher: Teacher, grad_loss, state, state_bytes: int, grad_short,
                      grad_stride: int, grad_alpha, grad_beta, stream=None) -> int:
    """``grad_short``: a tensor whose rows may be strided, or an address (``grad_stride`` elements a row)."""
    r = lib().dels_distill_grad(ctypes.byref(x), rows, V, ctypes.byref(teacher), _ptr(grad_loss), _ptr(state),
                                state_bytes, _row_ptr(grad_short), grad_stride, _ptr(grad_alpha), _ptr(grad_beta),
                                _stream(stream))
    if r == DELS_OK:
        _written(grad_short, grad_alpha, grad_beta)
    return r


def dels_distill_step(x: Rows, rows: int, V: int, teacher: Teacher, out_loss, grad_short, grad_stride: int,
                      grad_alpha, grad_beta, workspace, workspace_bytes: int, stream=None) -> int:
    r = lib().dels_distill_step(ctypes.byref(x), rows, V, ctypes.byref(teacher), _ptr(out_loss),
                                _row_ptr(grad_short), grad_stride, _ptr(grad_alpha), _ptr(grad_beta),
                                _ptr(workspace), workspace_bytes, _stream(stream))
    if r == DELS_OK:
        _written(out_loss, grad_short, grad_alpha, grad_beta)
    return r


def dels_profile_enable(on: bool) -> None:
    _check(lib().dels_profile_enable(1 if on else 0), "dels_profile_enable")


def dels_profile_reset() -> None:
    _check(lib().dels_profile_reset(), "dels_profile_reset")


def dels_profile_read(kernel_class: int):
    """(launches, total device ms) of one kernel class since the last reset."""
    n = ctypes.c_int(0)
    ms = ctypes.c_double(0.0)
    _check(lib().dels_profile_read(int(kernel_class), ctypes.byref(n), ctypes.byref(ms)), "dels_profile_read")
    return n.value, ms.value


# ----------------------------------------------------------------------------- conveniences

_KIND = {"gru": DELS_HEAD_GRU, "mlp": DELS_HEAD_MLP, "xfmr": DELS_HEAD_XFMR, "markov": DELS_HEAD_MARKOV}
_SLOTS = {
    "gru": ["w_ih", "w_hh", "w_rank", "input_table"],
    "mlp": ["w1", "w2"],
    "xfmr": ["pos", "wq", "wk", "wv", "wo", "w1", "w2"],
    "markov": [],
}


def make_head(spec, weights: Dict[str, torch.Tensor]) -> LocalHead:
    """LocalHead for a head spec (``kind``, ``wdtype``, dims) and a dict of device weight tensors
    (keys emb, w_vocab and the kind's slot names). The caller keeps the tensors alive."""
    h = LocalHead()
    h.kind = _KIND[spec.kind]
    h.wdtype = DELS_BF16 if spec.wdtype == "bf16" else DELS_F32
    h.d_model, h.d_hidden, h.d_rank = spec.d_model, spec.d_hidden, spec.d_rank
    h.window, h.n_layers, h.n_heads, h.max_pos = spec.window, spec.n_layers, spec.n_heads, spec.max_pos
    h.emb = _ptr(weights["emb"])
    h.w_vocab = _ptr(weights["w_vocab"])
    for i, name in enumerate(_SLOTS[spec.kind]):
        if name in weights:
            h.w[i] = _ptr(weights[name])
    return h


class Drafter:
    """One local head + one workspace for repeated dels_draft_block calls."""

    def __init__(self, spec, weights: Dict[str, torch.Tensor], B: int, n: int, V: int, device=None):
        self.spec, self.weights = spec, weights
        self.head = make_head(spec, weights)
        self.B, self.n, self.V = B, n, V
        self.device = device or weights["w_vocab"].device
        nbytes = dels_draft_workspace_bytes(self.head, B, n, V)
        if nbytes == 0:
            raise DelsError(-2, "dels_draft_workspace_bytes")
        self.ws_bytes = nbytes
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
        self.tokens = torch.empty(B, n, dtype=torch.int32, device=self.device)
        self.logprob = torch.empty(B, n, dtype=torch.float32, device=self.device)
        self.gap = torch.empty(B, n, dtype=torch.float32, device=self.device)

    def __call__(self, long_logits: torch.Tensor, log_prior: torch.Tensor, alpha, beta, stream=None):
        """``alpha``/``beta``: one weight for the block, or n per-position weights."""
        if hasattr(alpha, "__len__") or hasattr(beta, "__len__"):
            a = list(alpha) if hasattr(alpha, "__len__") else [alpha] * self.n
            b = list(beta) if hasattr(beta, "__len__") else [beta] * self.n
            _check(dels_draft_block_weighted(self.head, long_logits, dtype_code(long_logits), log_prior, a, b,
                                             self.B, self.n, self.V, self.tokens, self.logprob, self.gap,
                                             self.workspace, self.ws_bytes, stream), "dels_draft_block_weighted")
        else:
            _check(dels_draft_block(self.head, long_logits, dtype_code(long_logits), log_prior, alpha, beta, self.B,
                                    self.n, self.V, self.tokens, self.logprob, self.gap, self.workspace,
                                    self.ws_bytes, stream), "dels_draft_block")
        return self.tokens, self.logprob, self.gap

    def sample(self, long_logits: torch.Tensor, log_prior: torch.Tensor, alpha, beta, seed: int, step: int,
               stream=None):
        """Temperature-1 block: returns (tokens, logprob, key gap, draft state)."""
        a = list(alpha) if hasattr(alpha, "__len__") else [alpha] * self.n
        b = list(beta) if hasattr(beta, "__len__") else [beta] * self.n
        if getattr(self, "state", None) is None:
            self.state_bytes = dels_draft_state_bytes(self.head, self.B, self.n)
            self.state = torch.zeros(self.state_bytes, dtype=torch.uint8, device=self.device)
        _check(dels_draft_block_sampled(self.head, long_logits, dtype_code(long_logits), log_prior, a, b, self.B,
                                        self.n, self.V, seed, step, self.tokens, self.logprob, self.gap, self.state,
                                        self.state_bytes, self.workspace, self.ws_bytes, stream),
               "dels_draft_block_sampled")
        return self.tokens, self.logprob, self.gap, self.state

    def status(self, stream=None) -> int:
        return dels_read_status(self.workspace, stream)


# ----------------------------------------------------------------------------- scoring and distillation

def _row_ptr(x) -> Optional[int]:
    """Device address of [rows, V] logits whose rows may be strided."""
    if not isinstance(x, torch.Tensor):
        return _ptr(x)
    if not x.is_cuda:
        raise ValueError("expected a CUDA tensor: the library's entry points take device pointers")
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("expected [rows, V] logits whose rows are dense")
    return x.data_ptr()


def _row_stride(x: torch.Tensor, shape, what: str) -> int:
    """Elements from one row to the next (a single row's own length: its stride may be anything)."""
    rows, V = shape
    step, one = x.stride()
    if V > 1 and one != 1:
        raise ValueError(f"{what}: expected [rows, V] logits whose rows are dense")
    if rows <= 1:
        return V
    if step < V:
        raise ValueError(f"{what}: rows overlap")
    return step


def _of(t, dtype, shape, device: int, what) -> Optional[int]:
    """Device address of a dense tensor of this dtype and shape on this device."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} {list(shape)} on cuda:{device}, "
                         f"got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _logits(t, shape, dtype, device: int, what) -> int:
    """Device address of [rows, V] logits (their rows may be strided)."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"{what} must be {dtype} {list(shape)} on cuda:{device}, "
                         f"got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


_increment_version = torch._C._increment_version      # of an iterable of tensors


def _written(*tensors) -> None:
    """Tells the autograd engine that the library has written these (None, or an address: not known to it): a graph
    that still needs what they held then refuses its backward pass instead of taking what they hold now."""
    _increment_version([t for t in tensors if isinstance(t, torch.Tensor)])


def _outputs(device, *shapes):
    """Float32 outputs of these shapes in one buffer, and the buffer: its version, which is theirs too, is moved by
    every call that writes them."""
    sizes = [math.prod(shape) for shape in shapes]
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + (n + 63) // 64 * 64)
    buf = torch.empty(starts[-1], dtype=torch.float32, device=device)
    return [buf[i:i + n].view(shape) for i, n, shape in zip(starts, sizes, shapes)], buf


def rows_of(rows: int, V: int, long=None, short=None, log_prior=None, alpha=None, beta=None,
            temperature: float = 1.0) -> Rows:
    """``dels_rows`` of [rows, V] logit tensors (one dtype, rows may be strided), a
    [V] prior and [n_weights] fusion weights. The caller keeps the tensors alive."""
    one = long if long is not None else short
    if one is None:
        raise ValueError("rows need long or short logits")
    if not one.is_cuda:
        raise ValueError("expected a CUDA tensor: the library's entry points take device pointers")
    shape, dev, dtype = (rows, V), one.get_device(), one.dtype
    x = Rows()
    x.dtype = dtype_code(dtype)
    if long is not None:
        x.long_logits = _logits(long, shape, dtype, dev, "long")
        x.long_stride = _row_stride(long, shape, "long")
    if short is not None:
        x.short_logits = _logits(short, shape, dtype, dev, "short")
        x.short_stride = _row_stride(short, shape, "short")
    if log_prior is not None:
        x.log_prior = _of(log_prior, torch.float32, (V,), dev, "log_prior")
    if alpha is not None:
        x.n_weights = alpha.numel()
        x.alpha = _of(alpha, torch.float32, (x.n_weights,), dev, "alpha")
    if beta is not None:
        n = beta.numel()
        if alpha is not None and n != x.n_weights:
            raise ValueError("alpha and beta must have the same length")
        x.n_weights = n
        x.beta = _of(beta, torch.float32, (n,), dev, "beta")
    x.temperature = temperature
    return x


def teacher_of(rows: int, ids: torch.Tensor, logprob: torch.Tensor, row_weight=None, tail: bool = False) -> Teacher:
    """``dels_teacher`` of [rows, k] ids and log-probabilities. The caller keeps the tensors alive."""
    if ids.dim() != 2:
        raise ValueError("ids must be [rows, k]")
    if not ids.is_cuda:
        raise ValueError("expected a CUDA tensor: the library's entry points take device pointers")
    k, dev = ids.shape[1], ids.get_device()
    return Teacher(_of(ids, torch.int32, (rows, k), dev, "ids"), _of(logprob, torch.float32, (rows, k), dev, "logprob"),
                   k, 1 if tail else 0, _of(row_weight, torch.float32, (rows,), dev, "row_weight"))


def _device_index(device) -> int:
    device = torch.device(device or "cuda")
    if device.type != "cuda":
        raise ValueError("expected a CUDA device: the library's entry points take device pointers")
    return torch.cuda.current_device() if device.index is None else device.index


def _current_device() -> int:
    return torch._C._cuda_getDevice()


def _need_current(device: int) -> None:
    """The library launches on the current device: tensors of another one are refused before it sees them."""
    if _current_device() != device:
        raise ValueError(f"the tensors are on cuda:{device}, and the current device is cuda:{_current_device()}: "
                         f"call under torch.cuda.device({device})")


class TokenScorer:
    """Log-probabilities of given tokens, entropies and the ``top_k`` most likely
    entries of [rows, V] logits, plain or fused: outputs and a workspace for
    repeated ``dels_score_rows`` calls."""

    def __init__(self, rows: int, V: int, top_k: int = 0, device=None):
        self.rows, self.V, self.top_k = rows, V, top_k
        self._dev = _device_index(device)
        self.device = torch.device("cuda", self._dev)
        self.ws_bytes = dels_score_workspace_bytes(rows, V)
        if self.ws_bytes == 0:
            raise DelsError(DELS_ERR_BAD_SHAPE, "dels_score_workspace_bytes")
        self.workspace = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.top_ids = self.top_logprob = None
        if top_k > 0:
            out, buf = _outputs(self.device, (rows,), (rows,), (rows, top_k), (rows, top_k))
            self.top_ids, self.top_logprob = out[2].view(torch.int32), out[3]
        else:
            out, buf = _outputs(self.device, (rows,), (rows,))
        self.logprob, self.entropy = out[:2]
        self._writes = (buf,)
        self._call = lib().dels_score_rows
        self._own = [_ptr(t) for t in (self.logprob, self.entropy, self.top_ids, self.top_logprob, self.workspace)]

    def __call__(self, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, *, short=None, log_prior=None,
                 alpha=None, beta=None, temperature: float = 1.0, stream=None):
        """(log-probabilities or None without tokens, entropies, top ids, top log-probabilities)."""
        _need_current(self._dev)
        x = rows_of(self.rows, self.V, logits, short, log_prior, alpha, beta, temperature)
        if logits.get_device() != self._dev:
            raise ValueError(f"logits must be on {self.device}")
        tok = _of(tokens, torch.int32, (self.rows,), self._dev, "tokens")
        lp, ent, ids, tlp, ws = self._own
        r = self._call(ctypes.byref(x), self.rows, self.V, tok, self.top_k, lp if tok else None, ent, ids, tlp, ws,
                       self.ws_bytes, _stream(stream))
        if r != DELS_OK:
            raise DelsError(r, "dels_score_rows")
        _increment_version(self._writes)
        return self.logprob if tokens is not None else None, self.entropy, self.top_ids, self.top_logprob

    def status(self, stream=None) -> int:
        return dels_read_status(self.workspace, stream)


class Distiller:
    """Distillation of a local head's [rows, V] logits from ``k`` teacher entries a
    row: outputs, state and a workspace for repeated calls. ``n_weights``: fusion
    weights of the calls' alpha and beta."""

    def __init__(self, rows: int, V: int, k: int, dtype: torch.dtype, n_weights: int = 1, tail: bool = False,
                 temperature: float = 1.0, device=None):
        self.rows, self.V, self.k, self.dtype, self.n_weights = rows, V, k, dtype, n_weights
        self.tail, self.temperature = tail, temperature
        dtype_code(dtype)
        self._dev = _device_index(device)
        self.device = torch.device("cuda", self._dev)
        self.ws_bytes = dels_distill_workspace_bytes(rows, V)
        if self.ws_bytes == 0:
            raise DelsError(DELS_ERR_BAD_SHAPE, "dels_distill_workspace_bytes")
        self.workspace = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)
        (self._loss, *self._grad_w), self._buf = _outputs(self.device, (rows,), (n_weights,), (n_weights,))
        self._grad = self._state = None
        self._own = [_ptr(t) for t in (self._loss, *self._grad_w, self.workspace)]
        self._call = lib().dels_distill_step

    def _args(self, short, ids, logprob, long, log_prior, alpha, beta, row_weight):
        _need_current(self._dev)
        if short.dtype is not self.dtype or short.get_device() != self._dev or ids.get_device() != self._dev:
            raise ValueError(f"short must be {self.dtype} and all tensors on {self.device}")
        x = rows_of(self.rows, self.V, long, short, log_prior, alpha, beta, self.temperature)
        if x.n_weights not in (0, self.n_weights):
            raise ValueError(f"alpha and beta must have {self.n_weights} entries")
        t = teacher_of(self.rows, ids, logprob, row_weight, self.tail)
        if t.k != self.k:
            raise ValueError(f"ids must be [{self.rows}, {self.k}]")
        return x, t

    def loss(self, short, ids, logprob, *, long=None, log_prior=None, alpha=None, beta=None, row_weight=None,
             stream=None) -> torch.Tensor:
        """The rows' losses, float32 [rows]."""
        x, t = self._args(short, ids, logprob, long, log_prior, alpha, beta, row_weight)
        if self._state is None:
            self._state = torch.empty(dels_distill_state_bytes(self.rows), dtype=torch.uint8, device=self.device)
        r = lib().dels_distill_loss(ctypes.byref(x), self.rows, self.V, ctypes.byref(t), self._own[0],
                                    self._state.data_ptr(), self._state.numel(), self._own[3], self.ws_bytes,
                                    _stream(stream))
        if r != DELS_OK:
            raise DelsError(r, "dels_distill_loss")
        _increment_version((self._buf,))
        return self._loss

    def step(self, short, ids, logprob, *, long=None, log_prior=None, alpha=None, beta=None, row_weight=None,
             out=None, stream=None):
        """(losses, gradient of ``short``, of alpha, of beta) of the sum of the losses;
        the weights' are None where the call has none (beta's too without a prior).
        ``out``: where the gradient goes ([rows, V], ``short`` itself for in place)."""
        x, t = self._args(short, ids, logprob, long, log_prior, alpha, beta, row_weight)
        if out is None:
            if self._grad is None:
                self._grad = torch.empty(self.rows, self.V, dtype=self.dtype, device=self.device)
            out = self._grad
        shape = (self.rows, self.V)
        to = _logits(out, shape, self.dtype, self._dev, "out")
        loss, ga, gb, ws = self._own
        has_a, has_b = alpha is not None, beta is not None and log_prior is not None
        r = self._call(ctypes.byref(x), self.rows, self.V, ctypes.byref(t), loss, to, _row_stride(out, shape, "out"),
                       ga if has_a else None, gb if has_b else None, ws, self.ws_bytes, _stream(stream))
        if r != DELS_OK:
            raise DelsError(r, "dels_distill_step")
        _increment_version((self._buf, out))
        return self._loss, out, self._grad_w[0] if has_a else None, self._grad_w[1] if has_b else None

    def status(self, stream=None) -> int:
        return dels_read_status(self.workspace, stream)


def _distill_structs(short, alpha, beta, long, log_prior, ids, logprob, row_weight, tail, temperature):
    """``dels_rows`` and ``dels_teacher`` of a distillation's tensors, on one device."""
    if short.dim() != 2:
        raise ValueError("short must be [rows, V]")
    rows, V = short.shape
    if ids.get_device() != short.get_device():
        raise ValueError(f"ids must be on {short.device}")
    _need_current(short.get_device())
    return (rows_of(rows, V, long, short, log_prior, alpha, beta, temperature),
            teacher_of(rows, ids, logprob, row_weight, tail))


def _lies_at(x: Rows, t: Teacher, short, alpha, beta, long, log_prior, ids, logprob, row_weight) -> bool:
    """Whether the structures' addresses are those of these tensors."""
    return (short.data_ptr() == x.short_logits and ids.data_ptr() == t.ids and logprob.data_ptr() == t.logprob
            and (long is None or long.data_ptr() == x.long_logits)
            and (log_prior is None or log_prior.data_ptr() == x.log_prior)
            and (alpha is None or alpha.data_ptr() == x.alpha) and (beta is None or beta.data_ptr() == x.beta)
            and (row_weight is None or row_weight.data_ptr() == t.row_weight))


def _layout(short, long):
    return short.dtype, short.shape, short.stride(), None if long is None else long.stride()


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, short, alpha, beta, long, log_prior, ids, logprob, row_weight, tail, temperature):
        x, t = _distill_structs(short, alpha, beta, long, log_prior, ids, logprob, row_weight, tail, temperature)
        rows, V = short.shape
        dev = short.device
        loss = torch.empty(rows, dtype=torch.float32, device=dev)
        # the state, and a workspace whose status word is not read (flagged rows are NaN)
        call = lib()
        nbytes = call.dels_distill_state_bytes(rows)
        state = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
        at = state.data_ptr()
        r = call.dels_distill_loss(ctypes.byref(x), rows, V, ctypes.byref(t), loss.data_ptr(), at, nbytes, at + nbytes,
                                   256, _stream(None))
        if r != DELS_OK:
            raise DelsError(r, "dels_distill_loss")
        # the tensors, not their addresses: backward() sees whether they were changed since, and takes what
        # saved-tensor hooks give back in their place (checkpointing: rows made again, the first ones freed)
        ctx.save_for_backward(short, alpha, beta, long, log_prior, ids, logprob, row_weight, state)
        ctx.call = x, t, at, nbytes, _layout(short, long), tail, temperature
        return loss

    @staticmethod
    def backward(ctx, grad_loss):
        if torch.is_grad_enabled():
            raise RuntimeError("distill_loss is differentiable once")
        short, alpha, beta, long, log_prior, ids, logprob, row_weight, state = ctx.saved_tensors
        x, t, at, nbytes, layout, tail, temperature = ctx.call
        if not (state.data_ptr() == at and _layout(short, long) == layout
                and _lies_at(x, t, short, alpha, beta, long, log_prior, ids, logprob, row_weight)):
            x, t = _distill_structs(short, alpha, beta, long, log_prior, ids, logprob, row_weight, tail, temperature)
            at = _of(state, torch.uint8, (nbytes + 256,), short.get_device(), "the saved state")
        rows, V = short.shape
        grad = torch.empty(rows, V, dtype=short.dtype, device=short.device)
        ga = torch.empty_like(alpha) if alpha is not None and ctx.needs_input_grad[1] else None
        gb = torch.empty_like(beta) if beta is not None and log_prior is not None and ctx.needs_input_grad[2] else None
        if grad_loss.dtype is not torch.float32 or not grad_loss.is_contiguous():
            grad_loss = grad_loss.to(torch.float32).contiguous()
        r = lib().dels_distill_grad(ctypes.byref(x), rows, V, ctypes.byref(t), grad_loss.data_ptr(), at, nbytes,
                                    grad.data_ptr(), V, None if ga is None else ga.data_ptr(),
                                    None if gb is None else gb.data_ptr(), _stream(None))
        if r != DELS_OK:
            raise DelsError(r, "dels_distill_grad")
        return grad, ga, gb, None, None, None, None, None, None, None


def distill_loss(short, ids, logprob, *, long=None, log_prior=None, alpha=None, beta=None, row_weight=None,
                 tail: bool = False, temperature: float = 1.0) -> torch.Tensor:
    """Distillation losses [rows] of a local head's logits, differentiable (once) in
    ``short``, ``alpha`` and ``beta``, on the current stream. Rows flagged as
    non-finite have a loss of NaN. The other tensors have no gradient here: where the engine
    records, none of them may require one (``detach()`` them)."""
    if torch.is_grad_enabled():
        for name, t in (("logprob", logprob), ("long", long), ("log_prior", log_prior), ("row_weight", row_weight)):
            if t is not None and t.requires_grad:
                raise ValueError(f"distill_loss has no gradient of {name}: detach it")
    return _DistillLoss.apply(short, alpha, beta, long, log_prior, ids, logprob, row_weight, tail, temperature)
