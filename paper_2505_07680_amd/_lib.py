"""ctypes binding of libspecrouter.so (the verify-step C ABI).

Argument marshalling only: every function takes torch tensors that already
live on the HIP device, checks their shapes against each other, and passes
raw pointers, sizes and the current stream to the C entry point of the same
name. All arithmetic happens in the library's kernels. A missing library or
a non-zero return code raises.
"""

from __future__ import annotations

import ctypes
import os
import re

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libspecrouter.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
HEADERS = [os.path.join(INCLUDE, h) for h in ("specrouter.h", "specrouter_sched.h", "specrouter_probe.h")]

SR_OK, SR_EINVAL, SR_EUNSUPPORTED, SR_EWORKSPACE, SR_ELAUNCH, SR_ESCRATCH = 0, -1, -2, -3, -4, -5
SR_F32, SR_BF16 = 0, 1
SR_ST_GAMMA, SR_ST_KVLEN, SR_ST_TOKEN, SR_ST_UNIFORM, SR_ST_ROLLBACK_GROW, SR_ST_TIMEOUT, SR_ST_CHAIN = 1, 2, 4, 8, 16, 32, 64
SR_ST_POSITION = 128

_c_p = ctypes.c_void_p
_c_i = ctypes.c_int
_c_i64 = ctypes.c_int64
_c_sz = ctypes.c_size_t
_c_f = ctypes.c_float
_c_d = ctypes.c_double
_c_dp = ctypes.POINTER(ctypes.c_double)
_c_ip = ctypes.POINTER(ctypes.c_int32)

class SamplingParams(ctypes.Structure):
    """specrouter_sampling: temperature (0 = greedy), top_k (0), top_p (1)."""

    _fields_ = [("temperature", ctypes.c_float), ("top_k", ctypes.c_int), ("top_p", ctypes.c_float)]


_SIGNATURES = {
    "specrouter_abi_version": (_c_i, []),
    "specrouter_status_string": (ctypes.c_char_p, [_c_i]),
    "specrouter_verify_attention_workspace_size": (_c_sz, [_c_i] * 6),
    "specrouter_verify_attention": (
        _c_i,
        [_c_p] * 7 + [_c_i] * 6 + [_c_f, _c_p, _c_sz, _c_p, _c_p],
    ),
    "specrouter_verify_attention_window_workspace_size": (_c_sz, [_c_i] * 8),
    "specrouter_verify_attention_window": (
        _c_i,
        [_c_p] * 7 + [_c_i] * 9 + [_c_f, _c_p, _c_sz, _c_p, _c_p],
    ),
    "specrouter_verify_attention_kv4_workspace_size": (_c_sz, [_c_i] * 8),
    "specrouter_verify_attention_kv4": (
        _c_i,
        [_c_p] * 9 + [_c_i] * 9 + [_c_f, _c_p, _c_sz, _c_p, _c_p],
    ),
    "specrouter_accept_workspace_size": (_c_sz, [_c_i] * 4),
    "specrouter_accept_and_diverge": (
        _c_i,
        [_c_p, _c_i64, _c_p, _c_i64, _c_i] + [_c_p] * 13 + [_c_i] * 3 + [_c_p, _c_sz, _c_p, _c_p],
    ),
    "specrouter_accept_and_diverge_sampled": (
        _c_i,
        [_c_p, _c_i64, _c_p, _c_i64, _c_i] + [_c_p] * 13 + [_c_i] * 3
        + [ctypes.POINTER(SamplingParams), _c_p, _c_sz, _c_p, _c_p],
    ),
    "specrouter_accept_and_rollback": (
        _c_i,
        [_c_p, _c_i64, _c_p, _c_i64, _c_i] + [_c_p] * 13 + [_c_i] * 3
        + [ctypes.POINTER(SamplingParams), _c_p, _c_p, _c_p, _c_i, _c_p, _c_sz, _c_p, _c_p],
    ),
    "specrouter_accept_and_rollback_noalloc": (
        _c_i,
        [_c_p, _c_i64, _c_p, _c_i64, _c_i] + [_c_p] * 13 + [_c_i] * 3
        + [ctypes.POINTER(SamplingParams), _c_p, _c_p, _c_p, _c_i, _c_p, _c_p],
    ),
    "specrouter_rollback": (_c_i, [_c_p] * 4 + [_c_i, _c_i, _c_p, _c_p]),
    "specrouter_chain_window": (_c_i, [_c_p, _c_p, _c_i, _c_i, _c_i] + [_c_p] * 5),
    "specrouter_kv_append": (_c_i, [_c_p] * 8 + [_c_i] * 5 + [_c_p, _c_p]),
    "specrouter_kv_compact": (_c_i, [_c_p] * 4 + [_c_i] * 4 + [_c_p, _c_p]),
    "specrouter_qk_norm_rope": (
        _c_i,
        [_c_p, _c_i64, _c_p, _c_i64, _c_p, _c_p, _c_i, _c_f, _c_p, _c_i, _c_i, _c_i] + [_c_p] * 4 + [_c_i] * 5
        + [_c_p, _c_p],
    ),
    "specrouter_kv4_append": (_c_i, [_c_p, _c_i64, _c_p, _c_i64] + [_c_p] * 10 + [_c_i] * 5 + [_c_p, _c_p]),
    "specrouter_chain_consensus": (_c_i, [_c_p, _c_p, _c_p, _c_i, _c_p, _c_p, _c_i, _c_i] + [_c_p] * 6),
    "specrouter_hbm_read_probe": (_c_i, [_c_p, _c_sz, _c_p, _c_p]),
    # chain scheduler (host code; host pointers)
    "specrouter_sched_create": (_c_i, [_c_i, _c_dp, _c_i, _c_i, _c_i, _c_d, _c_d, _c_d, ctypes.POINTER(_c_p)]),
    "specrouter_sched_destroy": (None, [_c_p]),
    "specrouter_sched_observe_time": (_c_i, [_c_p, _c_i, _c_d]),
    "specrouter_sched_set_similarity": (_c_i, [_c_p, _c_i, _c_i, _c_d]),
    "specrouter_sched_observe_step": (_c_i, [_c_p, _c_i, _c_i, _c_i, _c_i, _c_ip, _c_ip,
                                             ctypes.POINTER(ctypes.c_float)]),
    "specrouter_sched_calibrate": (_c_i, [_c_p, _c_dp, _c_dp]),
    "specrouter_sched_metrics": (_c_i, [_c_p, _c_dp, _c_dp, _c_dp, ctypes.POINTER(_c_i)]),
    "specrouter_sched_effective_time": (_c_i, [_c_p, _c_ip, _c_i, _c_dp]),
    "specrouter_sched_optimal_chain": (_c_i, [_c_p, _c_ip, ctypes.POINTER(_c_i), _c_dp, ctypes.POINTER(_c_i)]),
}

_lib = None


def load() -> ctypes.CDLL:
    """Load the library (once). Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2505_07680_amd.build`"
            )
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def header_functions() -> list[str]:
    """Names of the functions declared in include/*.h."""
    names = set()
    for h in HEADERS:
        text = re.sub(r"/\*.*?\*/", "", open(h).read(), flags=re.S)
        names.update(re.findall(r"\b(specrouter_\w+)\s*\(", text))
    return sorted(names)


# A call on one short sequence is bound by the host: with a c_void_p object per
# pointer and a Stream object per call an accept call took 19 us and an attention
# call 11, with plain integers (which ctypes takes for a c_void_p) 15 and 8.

def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    """The current device's current stream, as an integer handle."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(rc: int, what: str) -> None:
    if rc != SR_OK:
        msg = load().specrouter_status_string(rc).decode()
        raise RuntimeError(f"{what} failed: {rc} ({msg})")


_INT32 = torch.int32
_BF16 = torch.bfloat16


def _dev(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("all tensors must be on the HIP device")


def _int32s(ts, names):
    for t, n in zip(ts, names):
        if t is not None and t.dtype is not _INT32:
            raise TypeError(f"{n} must be int32")


_ACCEPT_I32 = ("draft_tokens", "gamma", "kv_len", "accept_len", "out_tokens", "new_len")


def _i32(t, name):
    if t is not None and t.dtype is not _INT32:
        raise TypeError(f"{name} must be int32")


def logits_dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SR_F32
    if t.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return SR_BF16
    raise TypeError("logits must be float32 or bf16 (bfloat16 or 16-bit bit patterns)")


def specrouter_abi_version() -> int:
    return load().specrouter_abi_version()


def specrouter_status_string(code: int) -> str:
    return load().specrouter_status_string(code).decode()


def specrouter_verify_attention_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap) -> int:
    return load().specrouter_verify_attention_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap)


def specrouter_verify_attention(q, k_cache, v_cache, cache_mask, kv_len, gamma, out, scale,
                                workspace=None, status=None):
    """q [B, gmax+1, Hq, D] bf16; k/v [B, Hkv, L_cap, D] bf16; out [B, gmax+1, Hq, D] fp32."""
    _dev(q, k_cache, v_cache, cache_mask, kv_len, gamma, out, workspace, status)
    _i32(kv_len, "kv_len")
    _i32(gamma, "gamma")
    B, G1, Hq, D = q.shape
    Hkv, L_cap = k_cache.shape[1], k_cache.shape[2]
    if k_cache.shape != (B, Hkv, L_cap, D) or v_cache.shape != k_cache.shape:
        raise ValueError("k_cache/v_cache must be [B, Hkv, L_cap, D]")
    if out.shape != (B, G1, Hq, D) or out.dtype != torch.float32:
        raise ValueError("out must be fp32 [B, gamma_max+1, Hq, D]")
    if q.element_size() != 2 or k_cache.element_size() != 2 or v_cache.element_size() != 2:
        raise TypeError("q, k_cache, v_cache must hold bf16")
    for t in (q, k_cache, v_cache, out):
        if not t.is_contiguous():
            raise ValueError("q, k_cache, v_cache and out must be contiguous")
    if cache_mask is not None and (cache_mask.shape != (B, L_cap) or cache_mask.element_size() != 1
                                   or not cache_mask.is_contiguous()):
        raise ValueError("cache_mask must be u8 [B, L_cap]")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load().specrouter_verify_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(cache_mask), _ptr(kv_len), _ptr(gamma), _ptr(out),
        B, G1 - 1, Hq, Hkv, D, L_cap, float(scale), _ptr(workspace), ws_bytes, _ptr(status), _stream(),
    )
    _check(rc, "specrouter_verify_attention")
    return out


def specrouter_accept_workspace_size(B, gamma_max, V, logits_dtype) -> int:
    return load().specrouter_accept_workspace_size(B, gamma_max, V, logits_dtype)


def _row_view(t, rows, V, name):
    if t.dim() != 3 or t.shape[1] < rows or t.shape[2] != V or t.stride(2) != 1 or t.stride(1) != V:
        raise ValueError(f"{name} must be [B, >= {rows}, V] with contiguous rows")
    return t.stride(0)


def specrouter_accept_and_diverge(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample,
                                  kv_len, accept_len, out_tokens, new_len, accept_prob, p_tok,
                                  q_tok, kl, tv, workspace, status=None):
    """p_logits [B, gmax+1, V]; q_logits [B, gmax, V] (rows contiguous, batch stride free)."""
    _accept(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len, accept_len, out_tokens,
            new_len, accept_prob, p_tok, q_tok, kl, tv, workspace, status, None)


def specrouter_accept_and_diverge_sampled(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample,
                                          kv_len, accept_len, out_tokens, new_len, accept_prob, p_tok,
                                          q_tok, kl, tv, workspace, status=None, temperature=1.0, top_k=0,
                                          top_p=1.0):
    """As specrouter_accept_and_diverge under softmax(logits / temperature);
    temperature 0 is greedy decoding (u_accept and u_resample may be None)."""
    _accept(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len, accept_len, out_tokens,
            new_len, accept_prob, p_tok, q_tok, kl, tv, workspace, status,
            SamplingParams(float(temperature), int(top_k), float(top_p)))


def specrouter_accept_and_rollback(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len,
                                   accept_len, out_tokens, new_len, accept_prob, p_tok, q_tok, kl, tv,
                                   cache_kv_len, cache_mask, phys_len, workspace, status=None, temperature=1.0,
                                   L_cap=None, top_k=0, top_p=1.0):
    """specrouter_accept_and_diverge_sampled, then specrouter_rollback of
    cache_kv_len / cache_mask to the accepted lengths, in one call."""
    _dev(cache_kv_len, cache_mask, phys_len)
    _i32(cache_kv_len, "cache_kv_len")
    B = out_tokens.shape[0]
    if cache_kv_len.shape != (B,):
        raise ValueError("cache_kv_len must be [B]")
    if cache_mask is not None:
        if cache_mask.shape[0] != B or not cache_mask.is_contiguous():
            raise ValueError("cache_mask must be contiguous [B, L_cap]")
        L_cap = cache_mask.shape[1]
    if L_cap is None:
        raise ValueError("L_cap is required when cache_mask is None")
    _accept(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len, accept_len, out_tokens,
            new_len, accept_prob, p_tok, q_tok, kl, tv, workspace, status,
            SamplingParams(float(temperature), int(top_k), float(top_p)),
            rollback=(cache_kv_len, cache_mask, phys_len, int(L_cap)))


def specrouter_accept_and_rollback_noalloc(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len,
                                           accept_len, out_tokens, new_len, accept_prob, p_tok, q_tok, kl, tv,
                                           cache_kv_len, cache_mask, phys_len, status=None, temperature=1.0,
                                           L_cap=None, top_k=0, top_p=1.0):
    """specrouter_accept_and_rollback with the library's own fixed device
    array as the workspace (no workspace argument, nothing allocated)."""
    _dev(cache_kv_len, cache_mask, phys_len)
    _i32(cache_kv_len, "cache_kv_len")
    B = out_tokens.shape[0]
    if cache_kv_len.shape != (B,):
        raise ValueError("cache_kv_len must be [B]")
    if cache_mask is not None:
        if cache_mask.shape[0] != B or not cache_mask.is_contiguous():
            raise ValueError("cache_mask must be contiguous [B, L_cap]")
        L_cap = cache_mask.shape[1]
    if L_cap is None:
        raise ValueError("L_cap is required when cache_mask is None")
    _accept(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len, accept_len, out_tokens,
            new_len, accept_prob, p_tok, q_tok, kl, tv, None, status,
            SamplingParams(float(temperature), int(top_k), float(top_p)),
            rollback=(cache_kv_len, cache_mask, phys_len, int(L_cap)), noalloc=True)


def _accept(p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len, accept_len, out_tokens,
            new_len, accept_prob, p_tok, q_tok, kl, tv, workspace, status, sampling, rollback=None, noalloc=False):
    tensors = (p_logits, q_logits, draft_tokens, gamma, u_accept, u_resample, kv_len, accept_len,
               out_tokens, new_len, accept_prob, p_tok, q_tok, kl, tv, workspace, status)
    _dev(*tensors)
    _int32s((draft_tokens, gamma, kv_len, accept_len, out_tokens, new_len), _ACCEPT_I32)
    B, G1 = out_tokens.shape
    gmax = G1 - 1
    V = p_logits.shape[2]
    code = logits_dtype_code(p_logits)
    ps = _row_view(p_logits, G1, V, "p_logits")
    qs = 0
    if gmax > 0:
        if logits_dtype_code(q_logits) != code:
            raise TypeError("p_logits and q_logits must share a dtype")
        qs = _row_view(q_logits, gmax, V, "q_logits")
    if (u_resample is not None and u_resample.shape != (B, G1)) or (
            gmax > 0 and u_accept is not None and u_accept.shape != (B, gmax)):
        raise ValueError("u_accept [B, gmax] and u_resample [B, gmax+1] expected")
    shape = (B, gmax)
    for t in (accept_prob, p_tok, q_tok, kl, tv):
        if t is not None and (t.shape != shape or t.dtype is not torch.float32):
            raise ValueError("float outputs must be fp32 [B, gamma_max]")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    common = (_ptr(p_logits), ps, _ptr(q_logits), qs, code, _ptr(draft_tokens), _ptr(gamma),
              _ptr(u_accept), _ptr(u_resample), _ptr(kv_len), _ptr(accept_len), _ptr(out_tokens),
              _ptr(new_len), _ptr(accept_prob), _ptr(p_tok), _ptr(q_tok), _ptr(kl), _ptr(tv),
              B, gmax, V, None if sampling is None else ctypes.byref(sampling))
    if noalloc:
        rkv, rmask, rphys, L_cap = rollback
        rc = load().specrouter_accept_and_rollback_noalloc(*common, _ptr(rkv), _ptr(rmask), _ptr(rphys), L_cap,
                                                           _ptr(status), _stream())
        _check(rc, "specrouter_accept_and_rollback_noalloc")
        return
    if rollback is not None:
        rkv, rmask, rphys, L_cap = rollback
        rc = load().specrouter_accept_and_rollback(*common, _ptr(rkv), _ptr(rmask), _ptr(rphys), L_cap,
                                                   _ptr(workspace), ws_bytes, _ptr(status), _stream())
        _check(rc, "specrouter_accept_and_rollback")
        return
    rc = load().specrouter_accept_and_diverge_sampled(*common, _ptr(workspace), ws_bytes, _ptr(status), _stream())
    _check(rc, "specrouter_accept_and_diverge" + ("" if sampling is None else "_sampled"))


def specrouter_hbm_read_probe(buf, sink=None):
    """Stream the bytes of the contiguous device tensor `buf` once (the read
    bandwidth probe); `sink` is an optional one-element int32 device tensor."""
    _dev(buf, sink)
    if not buf.is_contiguous():
        raise ValueError("buf must be contiguous")
    rc = load().specrouter_hbm_read_probe(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream())
    _check(rc, "specrouter_hbm_read_probe")


def specrouter_rollback(kv_len, cache_mask, new_len, phys_len=None, status=None, L_cap=None):
    _dev(kv_len, cache_mask, new_len, phys_len, status)
    _i32(kv_len, "kv_len")
    _i32(new_len, "new_len")
    B = kv_len.shape[0]
    if cache_mask is not None:
        if cache_mask.shape[0] != B or not cache_mask.is_contiguous():
            raise ValueError("cache_mask must be contiguous [B, L_cap]")
        L_cap = cache_mask.shape[1]
    if L_cap is None:
        raise ValueError("L_cap is required when cache_mask is None")
    rc = load().specrouter_rollback(_ptr(kv_len), _ptr(cache_mask), _ptr(new_len), _ptr(phys_len),
                                    B, int(L_cap), _ptr(status), _stream())
    _check(rc, "specrouter_rollback")


def specrouter_chain_window(accept_len, out_tokens, gamma_cap, gamma_next, drafts_next, ctx_len=None,
                            kv_len_next=None):
    """accept_len [B], out_tokens [B, gmax+1] of the level below -> gamma_next [B],
    drafts_next [B, gamma_cap] (and kv_len_next [B] from ctx_len [B])."""
    _dev(accept_len, out_tokens, gamma_next, drafts_next, ctx_len, kv_len_next)
    for t, n in ((accept_len, "accept_len"), (out_tokens, "out_tokens"), (gamma_next, "gamma_next"),
                 (drafts_next, "drafts_next"), (ctx_len, "ctx_len"), (kv_len_next, "kv_len_next")):
        _i32(t, n)
    B, G1 = out_tokens.shape
    if drafts_next.shape != (B, gamma_cap) or gamma_next.shape != (B,) or accept_len.shape != (B,):
        raise ValueError("accept_len [B], gamma_next [B] and drafts_next [B, gamma_cap] expected")
    rc = load().specrouter_chain_window(_ptr(accept_len), _ptr(out_tokens), B, G1 - 1, int(gamma_cap),
                                        _ptr(ctx_len), _ptr(gamma_next), _ptr(drafts_next), _ptr(kv_len_next),
                                        _stream())
    _check(rc, "specrouter_chain_window")


def specrouter_chain_consensus(ctx_len, k_lower, out_lower, k_upper, out_upper, len_upper, len_lower, pending,
                               n_pending, status=None):
    """Rows each level keeps after a two-level verify and the pending tokens."""
    _dev(ctx_len, k_lower, out_lower, k_upper, out_upper, len_upper, len_lower, pending, n_pending, status)
    for t in (ctx_len, k_lower, out_lower, k_upper, out_upper, len_upper, len_lower, pending, n_pending):
        _i32(t, "chain tensor")
    B = ctx_len.shape[0]
    if pending.shape != (B, 2) or out_lower.shape[0] != B or out_upper.shape[0] != B:
        raise ValueError("pending [B, 2], out_lower [B, gl+1], out_upper [B, gu+1] expected")
    rc = load().specrouter_chain_consensus(_ptr(ctx_len), _ptr(k_lower), _ptr(out_lower), out_lower.shape[1] - 1,
                                           _ptr(k_upper), _ptr(out_upper), out_upper.shape[1] - 1, B,
                                           _ptr(len_upper), _ptr(len_lower), _ptr(pending), _ptr(n_pending),
                                           _ptr(status), _stream())
    _check(rc, "specrouter_chain_consensus")


def specrouter_kv_append(k_new, v_new, gamma, k_cache, v_cache, cache_mask, kv_len, shared_len=None, status=None):
    """k_new/v_new [B, gmax+1, Hkv, D] bf16 -> k_cache/v_cache [B, Hkv, L_cap, D] at each cursor."""
    _dev(k_new, v_new, gamma, k_cache, v_cache, cache_mask, kv_len, shared_len, status)
    _i32(gamma, "gamma")
    _i32(kv_len, "kv_len")
    B, G1, Hkv, D = k_new.shape
    L_cap = k_cache.shape[2]
    if v_new.shape != k_new.shape or k_cache.shape != (B, Hkv, L_cap, D) or v_cache.shape != k_cache.shape:
        raise ValueError("k_new/v_new [B, gmax+1, Hkv, D] and k_cache/v_cache [B, Hkv, L_cap, D] expected")
    for t in (k_new, v_new, k_cache, v_cache):
        if not t.is_contiguous() or t.element_size() != 2:
            raise ValueError("K/V tensors must be contiguous bf16")
    if cache_mask is not None and (cache_mask.shape != (B, L_cap) or not cache_mask.is_contiguous()):
        raise ValueError("cache_mask must be u8 [B, L_cap]")
    rc = load().specrouter_kv_append(_ptr(k_new), _ptr(v_new), _ptr(gamma), _ptr(k_cache), _ptr(v_cache),
                                     _ptr(cache_mask), _ptr(kv_len), _ptr(shared_len), B, G1 - 1, Hkv, D, L_cap,
                                     _ptr(status), _stream())
    _check(rc, "specrouter_kv_append")


def specrouter_kv_compact(k_cache, v_cache, cache_mask, kv_len, status=None):
    _dev(k_cache, v_cache, cache_mask, kv_len, status)
    _i32(kv_len, "kv_len")
    B, Hkv, L_cap, D = k_cache.shape
    if v_cache.shape != k_cache.shape or cache_mask.shape != (B, L_cap):
        raise ValueError("k_cache/v_cache [B, Hkv, L_cap, D] and cache_mask [B, L_cap] expected")
    for t in (k_cache, v_cache, cache_mask):
        if not t.is_contiguous():
            raise ValueError("cache tensors must be contiguous")
    rc = load().specrouter_kv_compact(_ptr(k_cache), _ptr(v_cache), _ptr(cache_mask), _ptr(kv_len), B, Hkv, D, L_cap,
                                      _ptr(status), _stream())
    _check(rc, "specrouter_kv_compact")


# The calls below make all their checks in one expression and look for the words
# only when it fails: with a function call per tensor they took the host 2 to 5 us
# more, which is what a call on one short sequence is bound by.

def _current():
    """The current device, whose stream a call goes to."""
    return torch._C._cuda_getDevice()


def _refuse(where, **wanted):
    """Raise, naming the first tensor that is not what a call wants: name=(tensor
    or None, shape or None, dtypes or None, contiguous)."""
    for name, (t, shape, dtypes, contiguous) in wanted.items():
        if t is None:
            continue
        if t.get_device() != where:
            raise ValueError(f"{name} must be on the current HIP device, as all tensors of a call")
        if dtypes is not None and t.dtype not in dtypes:
            raise TypeError(f"{name} must be one of {dtypes}, not {t.dtype}")
        if shape is not None and t.shape != shape:
            raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
        if contiguous and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    raise ValueError("the call's tensors do not fit each other, or a size is out of range")


def _vector(t, n, dtype, where):
    """t is not a contiguous [n] of this type on this device."""
    return t.shape != (n,) or t.dtype is not dtype or not t.is_contiguous() or t.get_device() != where


def _not_mask(t, B, L_cap, where):
    return t.shape != (B, L_cap) or t.dtype not in _BYTE or not t.is_contiguous() or t.get_device() != where


def _not_word(t, where):
    return t.dtype is not _INT32 or t.get_device() != where


_INT_MAX = 0x7fffffff  # (a C int: ctypes would drop the bits above)
_BYTE = (torch.uint8, torch.int8, torch.bool)
_OUT = (_BF16, torch.float32)


def _row_stride(t, rows, H, D, name):
    """Elements from one row of t [B, rows, H, D] to the next, one stride for the whole batch."""
    s0, s1, s2, s3 = t.stride()
    if s3 == 1 and s2 == D and s0 == rows * s1:
        return s1
    B = t.shape[0]
    if (D > 1 and s3 != 1) or (H > 1 and s2 != D) or (B > 1 and rows > 1 and s0 != rows * s1):
        raise ValueError(f"{name} must be [B, rows, H, D] with contiguous heads and evenly spaced rows")
    return s1 if rows > 1 else s0 if B > 1 else H * D


def _meets(out, size, x, stride, width, rows):
    """Whether the bytes [out, out + size) touch one of `rows` runs of `width` bytes that lie `stride` apart from x on."""
    i = max(0, (out - x - width) // max(stride, 1) + 1)  # the first run that ends behind out
    return i < rows and x + i * stride < out + size


def _apart(name, out, size, **others):
    """Raise where an output of `size` bytes meets another argument, name=(address, stride, width, rows)."""
    for other, rows in others.items():
        if _meets(out, size, *rows):
            raise ValueError(f"{name} must not overlap {other}")


def specrouter_qk_norm_rope(q, k, q_weight, k_weight, eps, rope_table, position, gamma, q_out, k_out,
                            interleaved=False, status=None):
    """q [B, rows, Hq, D] and k [B, rows, Hkv, D] bf16 (views of one projection
    may be passed) -> q_out, k_out of the same shapes: every head normed (where
    its weight [D] is not None) and rotated to its position. rope_table fp32
    [max_positions, rot_dim] as from rope_table()."""
    here = _current()
    B, rows, Hq, D = qs = q.shape
    Bk, rows_k, Hkv, Dk = ks = k.shape
    max_positions, rot = rope_table.shape
    w = q_weight if q_weight is not None else k_weight
    code = SR_BF16 if w is None or w.dtype is _BF16 else SR_F32
    if (not (q.get_device() == k.get_device() == rope_table.get_device() == position.get_device() == gamma.get_device()
             == q_out.get_device() == k_out.get_device() == here)
            or Bk != B or rows_k != rows or Dk != D or max_positions > _INT_MAX
            or not (q.dtype is k.dtype is q_out.dtype is k_out.dtype is _BF16)
            or q_out.shape != qs or k_out.shape != ks or not q_out.is_contiguous() or not k_out.is_contiguous()
            or not (position.dtype is gamma.dtype is _INT32) or position.numel() != B or gamma.numel() != B
            or position.dim() != 1 or gamma.dim() != 1 or not position.is_contiguous() or not gamma.is_contiguous()
            or rope_table.dtype is not torch.float32 or not rope_table.is_contiguous()
            or q_weight is not None and _vector(q_weight, D, w.dtype, here)
            or k_weight is not None and _vector(k_weight, D, w.dtype, here)
            or w is not None and w.dtype not in _OUT or status is not None and _not_word(status, here)):
        _refuse(here, q=(q, None, (_BF16,), False), k=(k, (B, rows, Hkv, D), (_BF16,), False),
                q_out=(q_out, qs, (_BF16,), True), k_out=(k_out, ks, (_BF16,), True),
                position=(position, (B,), (_INT32,), True), gamma=(gamma, (B,), (_INT32,), True),
                rope_table=(rope_table, None, (torch.float32,), True),
                q_weight=(q_weight, (D,), _OUT, True),
                k_weight=(k_weight, (D,), _OUT if q_weight is None else (w.dtype,), True), status=(status, None, (_INT32,), True))
    x, y, xo, yo = q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr()
    xs = Hq * D if q.is_contiguous() else _row_stride(q, rows, Hq, D, "q")
    ys = Hkv * D if k.is_contiguous() else _row_stride(k, rows, Hkv, D, "k")
    n = 2 * B * rows
    xe, ye, xoe, yoe = x + n * xs, y + n * ys, xo + n * Hq * D, yo + n * Hkv * D  # (past the last row of each)
    if (xo < xe and x < xoe and xo != x or xo < ye and y < xoe or yo < xe and x < yoe
            or yo < ye and y < yoe and yo != y or xo < yoe and yo < xoe):
        # (in place, where the library checks the strides: each its own rows, or those of both)
        ins = dict(q=(x, 2 * xs, 2 * Hq * D, B * rows), k=(y, 2 * ys, 2 * Hkv * D, B * rows))
        _apart("q_out", xo, xoe - xo, k_out=(yo, 1, yoe - yo, 1),
               **{i: v for i, v in ins.items() if xo != x or i == "k" and x != y})
        _apart("k_out", yo, yoe - yo, **{i: v for i, v in ins.items() if yo != y or i == "q" and x != y})
    rc = (_lib or load()).specrouter_qk_norm_rope(
        x, xs, y, ys, _ptr(q_weight), _ptr(k_weight), code, eps, rope_table.data_ptr(), max_positions, rot,
        1 if interleaved else 0, position.data_ptr(), gamma.data_ptr(), xo, yo, B, rows - 1, Hq, Hkv, D, _ptr(status),
        torch._C._cuda_getCurrentRawStream(here))
    if rc:
        _check(rc, "specrouter_qk_norm_rope")


def specrouter_kv4_append(k_new, v_new, gamma, k_codes, k_powers, v_codes, v_powers, cache_mask, kv_len,
                          shared_len=None, k_seen=None, v_seen=None, status=None):
    """k_new/v_new [B, rows, Hkv, D] bf16 -> the 4-bit cache (codes
    [B, Hkv, L_cap, D/2], powers [B, Hkv, L_cap, D/32], u8) at each cursor;
    k_seen/v_seen [B, rows, Hkv, D] bf16: the rows as the cache now holds them."""
    here = _current()
    B, rows, Hkv, D = ns = k_new.shape
    _, _, L_cap, _ = cs = k_codes.shape
    ps = k_powers.shape
    if (not (k_new.get_device() == v_new.get_device() == gamma.get_device() == kv_len.get_device()
             == k_codes.get_device() == k_powers.get_device() == v_codes.get_device() == v_powers.get_device() == here)
            or v_new.shape != ns or not (k_new.dtype is v_new.dtype is _BF16)
            or cs != (B, Hkv, L_cap, D // 2) or ps != (B, Hkv, L_cap, D // 32) or v_codes.shape != cs
            or v_powers.shape != ps
            or not (k_codes.dtype is k_powers.dtype is v_codes.dtype is v_powers.dtype is torch.uint8)
            or not (k_codes.is_contiguous() and k_powers.is_contiguous() and v_codes.is_contiguous()
                    and v_powers.is_contiguous() and gamma.is_contiguous() and kv_len.is_contiguous())
            or not (gamma.dtype is kv_len.dtype is _INT32) or gamma.numel() != B or kv_len.numel() != B
            or gamma.dim() != 1 or kv_len.dim() != 1
            or k_seen is not None and (k_seen.shape != ns or k_seen.dtype is not _BF16 or not k_seen.is_contiguous()
                                       or k_seen.get_device() != here)
            or v_seen is not None and (v_seen.shape != ns or v_seen.dtype is not _BF16 or not v_seen.is_contiguous()
                                       or v_seen.get_device() != here)
            or cache_mask is not None and _not_mask(cache_mask, B, L_cap, here)
            or shared_len is not None and _vector(shared_len, 1, _INT32, here)
            or status is not None and _not_word(status, here)):
        _refuse(here, k_new=(k_new, None, (_BF16,), False), v_new=(v_new, ns, (_BF16,), False),
                k_codes=(k_codes, (B, Hkv, L_cap, D // 2), (torch.uint8,), True),
                k_powers=(k_powers, (B, Hkv, L_cap, D // 32), (torch.uint8,), True),
                v_codes=(v_codes, (B, Hkv, L_cap, D // 2), (torch.uint8,), True),
                v_powers=(v_powers, (B, Hkv, L_cap, D // 32), (torch.uint8,), True),
                cache_mask=(cache_mask, (B, L_cap), _BYTE, True), gamma=(gamma, (B,), (_INT32,), True),
                kv_len=(kv_len, (B,), (_INT32,), True), shared_len=(shared_len, (1,), (_INT32,), True),
                k_seen=(k_seen, ns, (_BF16,), True), v_seen=(v_seen, ns, (_BF16,), True),
                status=(status, None, (_INT32,), True))
    x, y = k_new.data_ptr(), v_new.data_ptr()
    xs = Hkv * D if k_new.is_contiguous() else _row_stride(k_new, rows, Hkv, D, "k_new")
    ys = Hkv * D if v_new.is_contiguous() else _row_stride(v_new, rows, Hkv, D, "v_new")
    kc, kp, vc, vp = k_codes.data_ptr(), k_powers.data_ptr(), v_codes.data_ptr(), v_powers.data_ptr()
    ks = 0 if k_seen is None else k_seen.data_ptr()
    vs = 0 if v_seen is None else v_seen.data_ptr()
    if ks or vs:
        n, codes = 2 * B * rows, B * Hkv * L_cap * D // 2
        powers, size = codes // 16, n * Hkv * D
        xe, ye, kce, kpe, vce, vpe = x + n * xs, y + n * ys, kc + codes, kp + powers, vc + codes, vp + powers
        for o in (ks, vs):
            oe = o + size
            if (x < oe and o < xe and o != x or y < oe and o < ye and o != y or kc < oe and o < kce
                    or kp < oe and o < kpe or vc < oe and o < vce or vp < oe and o < vpe
                    or vs < oe and o < vs + size and o != vs):
                others = dict(k_new=(x, 2 * xs, 2 * Hkv * D, B * rows), v_new=(y, 2 * ys, 2 * Hkv * D, B * rows),
                              k_codes=(kc, 1, codes, 1), k_powers=(kp, 1, powers, 1), v_codes=(vc, 1, codes, 1),
                              v_powers=(vp, 1, powers, 1), v_seen=(vs, 1, size, 1))
                # (at the start of one of these: the library's to refuse, or in place)
                _apart("k_seen" if o == ks else "v_seen", o, size, **{i: v for i, v in others.items() if v[0] != o})
    rc = (_lib or load()).specrouter_kv4_append(
        x, xs, y, ys, gamma.data_ptr(), kc, kp, vc, vp, None if cache_mask is None else cache_mask.data_ptr(),
        kv_len.data_ptr(), None if shared_len is None else shared_len.data_ptr(), ks, vs, B, rows - 1, Hkv, D, L_cap, _ptr(status),
        torch._C._cuda_getCurrentRawStream(here))
    if rc:
        _check(rc, "specrouter_kv4_append")


def specrouter_verify_attention_window_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap, window, sinks) -> int:
    return load().specrouter_verify_attention_window_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap, window, sinks)


def specrouter_verify_attention_kv4_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap, window=0, sinks=0) -> int:
    return load().specrouter_verify_attention_kv4_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap, window, sinks)


def _bytes_of(workspace, here):
    if workspace is None:
        return 0
    if workspace.get_device() != here or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on the current HIP device")
    return workspace.numel() * workspace.element_size()


def specrouter_verify_attention_window(q, k_cache, v_cache, cache_mask, kv_len, gamma, out, scale, window, sinks=0,
                                       workspace=None, status=None):
    """specrouter_verify_attention where a row sees the last `window` cache rows
    up to its own and the first `sinks`; out [B, gmax+1, Hq, D] fp32 or bf16."""
    here = _current()
    B, G1, Hq, D = qs = q.shape
    Bk, Hkv, L_cap, Dk = cs = k_cache.shape
    out_bf16 = out.dtype is _BF16
    if (not (q.get_device() == k_cache.get_device() == v_cache.get_device() == kv_len.get_device()
             == gamma.get_device() == out.get_device() == here)
            or Bk != B or Dk != D or v_cache.shape != cs or out.shape != qs or not -_INT_MAX <= window <= _INT_MAX
            or not -_INT_MAX <= sinks <= _INT_MAX
            or not (q.dtype is k_cache.dtype is v_cache.dtype is _BF16)
            or not (out_bf16 or out.dtype is torch.float32)
            or not (q.is_contiguous() and k_cache.is_contiguous() and v_cache.is_contiguous() and out.is_contiguous()
                    and kv_len.is_contiguous() and gamma.is_contiguous())
            or not (gamma.dtype is kv_len.dtype is _INT32) or gamma.numel() != B or kv_len.numel() != B
            or gamma.dim() != 1 or kv_len.dim() != 1
            or cache_mask is not None and _not_mask(cache_mask, B, L_cap, here)
            or status is not None and _not_word(status, here)):
        _refuse(here, q=(q, None, (_BF16,), True), k_cache=(k_cache, (B, Hkv, L_cap, D), (_BF16,), True),
                v_cache=(v_cache, (B, Hkv, L_cap, D), (_BF16,), True), cache_mask=(cache_mask, (B, L_cap), _BYTE, True),
                kv_len=(kv_len, (B,), (_INT32,), True), gamma=(gamma, (B,), (_INT32,), True),
                out=(out, qs, _OUT, True), status=(status, None, (_INT32,), True))
    rc = (_lib or load()).specrouter_verify_attention_window(
        q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), _ptr(cache_mask), kv_len.data_ptr(), gamma.data_ptr(),
        out.data_ptr(), SR_BF16 if out_bf16 else SR_F32, B, G1 - 1, Hq, Hkv, D, L_cap, window, sinks, scale,
        _ptr(workspace), _bytes_of(workspace, here), _ptr(status), torch._C._cuda_getCurrentRawStream(here))
    if rc:
        _check(rc, "specrouter_verify_attention_window")
    return out


def specrouter_verify_attention_kv4(q, k_codes, k_powers, v_codes, v_powers, cache_mask, kv_len, gamma, out, scale,
                                    window=0, sinks=0, workspace=None, status=None):
    """The attention over a 4-bit cache (codes [B, Hkv, L_cap, D/2], powers
    [B, Hkv, L_cap, D/32], u8), of all keys (window 0) or a window and sinks;
    out [B, gmax+1, Hq, D] fp32 or bf16."""
    here = _current()
    B, G1, Hq, D = qs = q.shape
    _, Hkv, L_cap, _ = cs = k_codes.shape
    ps = k_powers.shape
    out_bf16 = out.dtype is _BF16
    if (not (q.get_device() == k_codes.get_device() == k_powers.get_device() == v_codes.get_device()
             == v_powers.get_device() == kv_len.get_device() == gamma.get_device() == out.get_device() == here)
            or cs != (B, Hkv, L_cap, D // 2) or ps != (B, Hkv, L_cap, D // 32) or v_codes.shape != cs
            or v_powers.shape != ps or out.shape != qs or q.dtype is not _BF16 or not -_INT_MAX <= window <= _INT_MAX
            or not -_INT_MAX <= sinks <= _INT_MAX
            or not (k_codes.dtype is k_powers.dtype is v_codes.dtype is v_powers.dtype is torch.uint8)
            or not (out_bf16 or out.dtype is torch.float32)
            or not (q.is_contiguous() and k_codes.is_contiguous() and k_powers.is_contiguous()
                    and v_codes.is_contiguous() and v_powers.is_contiguous() and out.is_contiguous()
                    and kv_len.is_contiguous() and gamma.is_contiguous())
            or not (gamma.dtype is kv_len.dtype is _INT32) or gamma.numel() != B or kv_len.numel() != B
            or gamma.dim() != 1 or kv_len.dim() != 1
            or cache_mask is not None and _not_mask(cache_mask, B, L_cap, here)
            or status is not None and _not_word(status, here)):
        _refuse(here, q=(q, None, (_BF16,), True), k_codes=(k_codes, (B, Hkv, L_cap, D // 2), (torch.uint8,), True),
                k_powers=(k_powers, (B, Hkv, L_cap, D // 32), (torch.uint8,), True),
                v_codes=(v_codes, (B, Hkv, L_cap, D // 2), (torch.uint8,), True),
                v_powers=(v_powers, (B, Hkv, L_cap, D // 32), (torch.uint8,), True),
                cache_mask=(cache_mask, (B, L_cap), _BYTE, True), kv_len=(kv_len, (B,), (_INT32,), True),
                gamma=(gamma, (B,), (_INT32,), True), out=(out, qs, _OUT, True), status=(status, None, (_INT32,), True))
    rc = (_lib or load()).specrouter_verify_attention_kv4(
        q.data_ptr(), k_codes.data_ptr(), k_powers.data_ptr(), v_codes.data_ptr(), v_powers.data_ptr(),
        _ptr(cache_mask), kv_len.data_ptr(), gamma.data_ptr(), out.data_ptr(), SR_BF16 if out_bf16 else SR_F32, B,
        G1 - 1, Hq, Hkv, D, L_cap, window, sinks, scale, _ptr(workspace), _bytes_of(workspace, here), _ptr(status),
        torch._C._cuda_getCurrentRawStream(here))
    if rc:
        _check(rc, "specrouter_verify_attention_kv4")
    return out


# ----------------------------------------------------------------------------
# Buffer helpers (allocation only).

def rope_table(max_positions, rot_dim, theta=10000.0, device="cuda"):
    """fp32 [max_positions, rot_dim] for specrouter_qk_norm_rope: the cosines,
    then the sines, of t * theta^(-2 n / rot_dim), n < rot_dim / 2, at every
    position t (angles in 64 bits: at far positions 32 would lose them)."""
    n = torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device)
    t = torch.arange(max_positions, dtype=torch.float64, device=device)
    angle = t[:, None] * theta ** (-n / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], -1).float()


class Kv4Cache:
    """An empty 4-bit K/V cache: k_codes, k_powers, v_codes, v_powers."""

    def __init__(self, B: int, Hkv: int, L_cap: int, D: int, device="cuda"):
        u8 = dict(dtype=torch.uint8, device=device)
        self.k_codes = torch.zeros(B, Hkv, L_cap, D // 2, **u8)
        self.k_powers = torch.zeros(B, Hkv, L_cap, D // 32, **u8)
        self.v_codes = torch.zeros(B, Hkv, L_cap, D // 2, **u8)
        self.v_powers = torch.zeros(B, Hkv, L_cap, D // 32, **u8)


class AcceptBuffers:
    """Outputs and the self-resetting workspace of one accept-and-diverge call shape."""

    def __init__(self, B: int, gamma_max: int, V: int, logits_dtype: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.accept_len = torch.empty(B, **i32)
        self.out_tokens = torch.empty(B, gamma_max + 1, **i32)
        self.new_len = torch.empty(B, **i32)
        self.accept_prob = torch.empty(B, gamma_max, **f32)
        self.p_tok = torch.empty(B, gamma_max, **f32)
        self.q_tok = torch.empty(B, gamma_max, **f32)
        self.kl = torch.empty(B, gamma_max, **f32)
        self.tv = torch.empty(B, gamma_max, **f32)
        n = specrouter_accept_workspace_size(B, gamma_max, V, logits_dtype)
        if n == 0:
            raise RuntimeError("accept workspace query failed")
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=device)  # zero before first use
        self.status = torch.zeros(1, **i32)


def attention_workspace(B, gamma_max, Hq, Hkv, D, L_cap, device="cuda"):
    n = specrouter_verify_attention_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap)
    return None if n == 0 else torch.zeros(n, dtype=torch.uint8, device=device)


def attention_window_workspace(B, gamma_max, Hq, Hkv, D, L_cap, window, sinks=0, device="cuda"):
    n = specrouter_verify_attention_window_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap, window, sinks)
    return None if n == 0 else torch.zeros(n, dtype=torch.uint8, device=device)


def attention_kv4_workspace(B, gamma_max, Hq, Hkv, D, L_cap, window=0, sinks=0, device="cuda"):
    n = specrouter_verify_attention_kv4_workspace_size(B, gamma_max, Hq, Hkv, D, L_cap, window, sinks)
    return None if n == 0 else torch.zeros(n, dtype=torch.uint8, device=device)


# ----------------------------------------------------------------------------
# Chain scheduler (host code). Inputs are copied into host arrays; the
# arithmetic is the library's.

def _host(t, dtype):
    """A contiguous host numpy array of `t` (a torch tensor on any device, or
    array-like) with the given numpy dtype."""
    import numpy as np

    if isinstance(t, torch.Tensor):
        t = t.detach().cpu().numpy()
    return np.ascontiguousarray(np.asarray(t), dtype=dtype)


def _as_ptr(a, ctype):
    return a.ctypes.data_as(ctypes.POINTER(ctype))


def specrouter_sched_create(capability, target, window, max_levels=None, ema_time=0.2, ema_sim=0.1,
                            prior_weight=1.0):
    import numpy as np

    cap = _host(capability, np.float64)
    n = int(cap.shape[0])
    h = ctypes.c_void_p()
    rc = load().specrouter_sched_create(n, _as_ptr(cap, ctypes.c_double), int(target), int(window),
                                        n if max_levels is None else int(max_levels), float(ema_time),
                                        float(ema_sim), float(prior_weight), ctypes.byref(h))
    _check(rc, "specrouter_sched_create")
    return h


def specrouter_sched_destroy(handle) -> None:
    load().specrouter_sched_destroy(handle)


def specrouter_sched_observe_time(handle, model, seconds_per_token) -> None:
    _check(load().specrouter_sched_observe_time(handle, int(model), float(seconds_per_token)),
           "specrouter_sched_observe_time")


def specrouter_sched_set_similarity(handle, draft, verifier, simscore) -> None:
    _check(load().specrouter_sched_set_similarity(handle, int(draft), int(verifier), float(simscore)),
           "specrouter_sched_set_similarity")


def specrouter_sched_observe_step(handle, draft, verifier, gamma, accept_len, tv) -> None:
    """gamma [B], accept_len [B], tv [B, gamma_max]: the accept call's outputs
    (device tensors are copied to the host)."""
    import numpy as np

    g = _host(gamma, np.int32)
    k = _host(accept_len, np.int32)
    t = _host(tv, np.float32)
    if t.ndim != 2 or g.shape != (t.shape[0],) or k.shape != g.shape:
        raise ValueError("gamma [B], accept_len [B] and tv [B, gamma_max] expected")
    rc = load().specrouter_sched_observe_step(handle, int(draft), int(verifier), int(t.shape[0]), int(t.shape[1]),
                                              _as_ptr(g, ctypes.c_int32), _as_ptr(k, ctypes.c_int32),
                                              _as_ptr(t, ctypes.c_float))
    _check(rc, "specrouter_sched_observe_step")


def specrouter_sched_calibrate(handle):
    A, B = ctypes.c_double(), ctypes.c_double()
    _check(load().specrouter_sched_calibrate(handle, ctypes.byref(A), ctypes.byref(B)), "specrouter_sched_calibrate")
    return A.value, B.value


def specrouter_sched_metrics(handle, n_models):
    """(T [n], SimScore [n, n], (A, B), number of kept observations)."""
    import numpy as np

    T = np.empty(n_models, np.float64)
    S = np.empty((n_models, n_models), np.float64)
    c = np.empty(2, np.float64)
    n_obs = ctypes.c_int()
    _check(load().specrouter_sched_metrics(handle, _as_ptr(T, ctypes.c_double), _as_ptr(S, ctypes.c_double),
                                           _as_ptr(c, ctypes.c_double), ctypes.byref(n_obs)),
           "specrouter_sched_metrics")
    return T, S, (float(c[0]), float(c[1])), n_obs.value


def specrouter_sched_effective_time(handle, chain) -> float:
    import numpy as np

    c = _host(chain, np.int32)
    t = ctypes.c_double()
    _check(load().specrouter_sched_effective_time(handle, _as_ptr(c, ctypes.c_int32), int(c.shape[0]),
                                                  ctypes.byref(t)), "specrouter_sched_effective_time")
    return t.value


def specrouter_sched_optimal_chain(handle, n_models):
    """(chain as a list of model indices, predicted T_eff, number of candidates)."""
    import numpy as np

    out = np.empty(n_models, np.int32)
    n, cnt = ctypes.c_int(), ctypes.c_int()
    t = ctypes.c_double()
    _check(load().specrouter_sched_optimal_chain(handle, _as_ptr(out, ctypes.c_int32), ctypes.byref(n),
                                                 ctypes.byref(t), ctypes.byref(cnt)),
           "specrouter_sched_optimal_chain")
    return out[:n.value].tolist(), t.value, cnt.value


class ChainScheduler:
    """Owning wrapper of a scheduler handle (Section 4.2, Algorithm 1)."""

    def __init__(self, capability, target, window, max_levels=None, ema_time=0.2, ema_sim=0.1,
                 prior_weight=1.0):
        self.n = len(capability)
        self.handle = specrouter_sched_create(capability, target, window, max_levels, ema_time, ema_sim,
                                              prior_weight)

    def close(self):
        if self.handle is not None:
            specrouter_sched_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def observe_time(self, model, seconds_per_token):
        specrouter_sched_observe_time(self.handle, model, seconds_per_token)

    def set_similarity(self, draft, verifier, simscore):
        specrouter_sched_set_similarity(self.handle, draft, verifier, simscore)

    def observe_step(self, draft, verifier, gamma, accept_len, tv):
        specrouter_sched_observe_step(self.handle, draft, verifier, gamma, accept_len, tv)

    def calibrate(self):
        return specrouter_sched_calibrate(self.handle)

    def metrics(self):
        return specrouter_sched_metrics(self.handle, self.n)

    def effective_time(self, chain):
        return specrouter_sched_effective_time(self.handle, chain)

    def optimal_chain(self):
        return specrouter_sched_optimal_chain(self.handle, self.n)
