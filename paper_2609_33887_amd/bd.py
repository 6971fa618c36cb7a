"""ctypes binding of ``libbd.so`` (argument marshalling only).

The functions keep the C names and argument order of ``include/bd.h``; device
pointers are plain integers (``tensor.data_ptr()``).  PyTorch is used by the
helpers at the bottom only to allocate device memory and to name the stream.
No computation of the decoding path happens in Python, and there is no
fallback: importing this module fails loudly when the library is missing.
"""
from __future__ import annotations

import ctypes
import os
from typing import Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbd.so")

BD_OK, BD_EINVAL, BD_ENOMEM, BD_EHIP, BD_ESTATE, BD_EUNSUPPORTED = 0, -1, -2, -3, -4, -5
BD_F32, BD_BF16 = 0, 1

EXPORTED = ["bd_init_model", "bd_model_kv_cache", "bd_quantize_fp8", "bd_quantize_mxfp4", "bd_prefill", "bd_denoise_step", "bd_commit", "bd_state_read",
            "bd_decode", "bd_decode_static", "bd_state_reset", "bd_state_steps", "bd_state_stats", "bd_profile",
            "bd_profile_read", "bd_plan_projection", "bd_kv_pages", "bd_kv_store", "bd_kv_read", "bd_kv_attention",
            "bd_kv_attention_workspace", "bd_token_scores", "bd_token_scores_workspace", "bd_state_free", "bd_model_free", "bd_last_error", "rl_risk_select",
            "rl_select", "rl_alpha_sweep", "rl_split_exceedance", "rl_monte_carlo"]
RL_METHODS = {"holm": 0, "bonferroni": 1, "fixed_sequence": 2, "uncorrected": 3, "plugin": 4}
# "rope" counts the coding of K and V into 8-bit pages; without them RoPE and the cache write are part of gemm_qkv
PROF_KINDS = ["embed", "norm", "gemm_qkv", "rope", "attn", "gemm_o", "gemm_gu", "gemm_down", "lm_head",
              "commit", "moe_route"]


class bd_model_cfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim",
                                              "ffn_dim", "vocab", "n_experts", "top_k", "expert_ffn",
                                              "n_shared")] + \
               [("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float), ("logit_scale", ctypes.c_float),
                ("mask_id", ctypes.c_int32), ("dtype", ctypes.c_int32), ("wq", ctypes.c_int32)]


BD_WQ_NONE, BD_WQ_FP8, BD_WQ_MXFP4 = 0, 1, 2
WQ = {None: BD_WQ_NONE, "bf16": BD_WQ_NONE, "fp8": BD_WQ_FP8, "mxfp4": BD_WQ_MXFP4}
MX_BLOCK = 32
BD_KV_PAIR, BD_KV_FP8 = 0, 1


class bd_decode_cfg(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("n_inflight", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("tau_semi", ctypes.c_float), ("tau_add", ctypes.c_float), ("skip_masked", ctypes.c_int32)]


def decode_cfg(tau: float, n_inflight: int, block_size: int, tau_semi=None, tau_add: float = 0.0,
               skip_masked: bool = False):
    """The C configuration; ``tau_semi=None`` switches semi-completion off."""
    return bd_decode_cfg(tau=tau, n_inflight=n_inflight, block_size=block_size,
                         tau_semi=-1.0 if tau_semi is None else tau_semi, tau_add=tau_add,
                         skip_masked=1 if skip_masked else 0)


class bd_kv_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "n_kv_heads", "head_dim", "page_size")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


STAT_NAMES = ("forwards", "rows", "lm_rows", "pairs", "keys", "committed", "active_forwards",
              "zero_commit", "static_saved", "static_deferred", "cache_writes", "skipped")


class BDError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"bd status {status}: {msg}")
        self.status = status


def _load():
    # torch ships its own libamdhip64; load it first so that libbd.so binds to
    # the same HIP runtime instance instead of pulling in a second one.
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_33887_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    sig = {
        "bd_init_model": [P(bd_model_cfg), P(VP), I32, VP, P(VP)],
        "bd_quantize_fp8": [VP, I32, I32, VP, VP, VP],
        "bd_quantize_mxfp4": [VP, I32, I32, I32, VP, VP, VP],
        "bd_model_kv_cache": [VP, I32, I32],
        "bd_prefill": [VP, VP, I32, I32, I32, P(bd_decode_cfg), P(VP)],
        "bd_denoise_step": [VP, VP, VP, VP, VP],
        "bd_commit": [VP, VP, P(I32)],
        "bd_state_read": [VP, VP, VP, VP, VP],
        "bd_decode": [VP, VP, I32, I32, I32, P(bd_decode_cfg), VP, VP, VP],
        "bd_decode_static": [VP, VP, I32, I32, I32, P(bd_decode_cfg), VP, VP, VP],
        "bd_state_reset": [VP, VP],
        "bd_state_steps": [VP, P(I32)],
        "bd_state_stats": [VP, VP, P(ctypes.c_int64), I32],
        "bd_profile": [VP, I32],
        "bd_profile_read": [VP, P(ctypes.c_double), P(I32)],
        "bd_plan_projection": [I32, I32, I32, I32, P(I32), P(I32), P(I32), P(ctypes.c_int64)],
        "bd_kv_pages": [I32, I32, I32, I32, VP, VP, VP, VP, VP, VP, I32, VP, VP, VP, VP, VP],
        "bd_kv_store": [P(bd_kv_cache), VP, VP, I32, I64, I64, I32, I32, VP, I32, VP, VP, VP],
        "bd_kv_read": [P(bd_kv_cache), VP, VP, I32, I64, I64, I32, I32, VP, I32, VP, VP, VP],
        "bd_kv_attention": [P(bd_kv_cache), VP, VP, I32, I64, I64, I32, I32, I32, I32, VP, I32, VP, VP, VP, I32,
                            ctypes.c_float, VP, I64, VP],
        "bd_kv_attention_workspace": [I32, I32, I32, I32, I32, I32, I32, I32, P(I64)],
        "bd_token_scores": [VP, I32, I64, I32, I32, I32, VP, VP, I32, I32, VP, VP, VP, VP, VP, I64, VP],
        "bd_token_scores_workspace": [I32, I32, I32, P(I64)],
        "bd_state_free": [VP],
        "bd_model_free": [VP],
        "rl_risk_select": [I32, I32, I32, P(ctypes.c_uint8), P(ctypes.c_double), ctypes.c_double,
                           ctypes.c_double, P(I32), P(ctypes.c_double), P(ctypes.c_uint8), P(I32), P(I32)],
        "rl_select": [I32, I32, I32, P(ctypes.c_uint8), P(ctypes.c_uint8), P(ctypes.c_double),
                      ctypes.c_double, ctypes.c_double, I32, P(I32), P(I32), P(ctypes.c_double),
                      P(ctypes.c_uint8), P(I32)],
        "rl_alpha_sweep": [I32, I32, I32, P(ctypes.c_uint8), P(ctypes.c_double), P(ctypes.c_double), I32,
                           ctypes.c_double, I32, P(I32), P(I32), P(I32), P(ctypes.c_double)],
        "rl_split_exceedance": [I32, I32, I32, P(ctypes.c_uint8), P(ctypes.c_double), ctypes.c_double,
                                ctypes.c_double, I32, P(I32), I32, P(ctypes.c_uint8), P(I32), P(I32),
                                P(I32), P(ctypes.c_double)],
        "rl_monte_carlo": [I32, I32, P(ctypes.c_double), ctypes.c_double, ctypes.c_double, I32, P(I32),
                           I32, I32, P(ctypes.c_double), P(I32), P(I32)],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = I32
    lib.bd_last_error.argtypes = []
    lib.bd_last_error.restype = ctypes.c_char_p
    return lib


lib = _load()


def bd_last_error() -> str:
    return lib.bd_last_error().decode()


def _check(st: int):
    if st != BD_OK:
        raise BDError(st, bd_last_error())


# ---------------------------------------------------------------- thin wrappers
def bd_init_model(cfg: bd_model_cfg, weight_ptrs: Sequence[int], stream: int = 0) -> int:
    arr = (ctypes.c_void_p * len(weight_ptrs))(*weight_ptrs)
    out = ctypes.c_void_p()
    _check(lib.bd_init_model(ctypes.byref(cfg), arr, len(weight_ptrs), ctypes.c_void_p(stream),
                             ctypes.byref(out)))
    return out.value


def bd_quantize_fp8(w_ptr: int, rows: int, cols: int, codes_ptr: int, scale_ptr: int, stream: int = 0):
    _check(lib.bd_quantize_fp8(w_ptr, rows, cols, codes_ptr, scale_ptr, ctypes.c_void_p(stream)))


def quantize_fp8(w_bf16_bits, device: str = "cuda:0"):
    """fp8 E4M3 codes and row scales of a bf16 matrix given as uint16 bit
    patterns [rows][cols] (numpy); returns numpy (codes uint8, scale float32)."""
    import numpy as np
    import torch
    a = np.ascontiguousarray(w_bf16_bits)
    rows, cols = a.shape
    w = torch.from_numpy(a.view(np.int16)).to(device)
    codes = torch.empty((rows, cols), dtype=torch.uint8, device=device)
    scale = torch.empty((rows,), dtype=torch.float32, device=device)
    bd_quantize_fp8(w.data_ptr(), rows, cols, codes.data_ptr(), scale.data_ptr(),
                    torch.cuda.current_stream(device).cuda_stream)
    torch.cuda.synchronize(device)
    return codes.cpu().numpy(), scale.cpu().numpy()


def bd_quantize_mxfp4(w_ptr: int, rows: int, cols: int, group_rows: int, codes_ptr: int, exps_ptr: int,
                      stream: int = 0):
    _check(lib.bd_quantize_mxfp4(w_ptr, rows, cols, group_rows, codes_ptr, exps_ptr, ctypes.c_void_p(stream)))


def quantize_mxfp4(w_bf16_bits, group_rows=None, device: str = "cuda:0"):
    """MXFP4 codes and block exponents of a bf16 matrix given as uint16 bit
    patterns [rows][cols] (numpy), in the library's layout (see
    bd_quantize_mxfp4); returns numpy (codes uint8 [groups][cols/32][group_rows][16],
    exps uint8 [groups][cols/32][group_rows])."""
    import numpy as np
    import torch
    a = np.ascontiguousarray(w_bf16_bits)
    rows, cols = a.shape
    gr = rows if group_rows is None else group_rows
    w = torch.from_numpy(a.view(np.int16)).to(device)
    nb = cols // MX_BLOCK
    codes = torch.empty((rows // gr, nb, gr, 16), dtype=torch.uint8, device=device)
    exps = torch.empty((rows // gr, nb, gr), dtype=torch.uint8, device=device)
    bd_quantize_mxfp4(w.data_ptr(), rows, cols, gr, codes.data_ptr(), exps.data_ptr(),
                      torch.cuda.current_stream(device).cuda_stream)
    torch.cuda.synchronize(device)
    return codes.cpu().numpy(), exps.cpu().numpy()


def bd_model_kv_cache(model: int, kind: int, page_size: int = 0):
    _check(lib.bd_model_kv_cache(model, kind, page_size))


def bd_prefill(model: int, prompt_ptr: int, b: int, P: int, G: int, cfg: bd_decode_cfg) -> int:
    out = ctypes.c_void_p()
    _check(lib.bd_prefill(model, prompt_ptr, b, P, G, ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def bd_denoise_step(model: int, state: int, conf_ptr: int = 0, tok_ptr: int = 0, logits_ptr: int = 0):
    _check(lib.bd_denoise_step(model, state, conf_ptr or None, tok_ptr or None, logits_ptr or None))


def bd_commit(model: int, state: int, want_done: bool = False):
    if want_done:
        d = ctypes.c_int32(0)
        _check(lib.bd_commit(model, state, ctypes.byref(d)))
        return bool(d.value)
    _check(lib.bd_commit(model, state, None))
    return None


def bd_state_read(model: int, state: int, tokens_ptr: int = 0, commit_ptr: int = 0, fwd_ptr: int = 0):
    _check(lib.bd_state_read(model, state, tokens_ptr or None, commit_ptr or None, fwd_ptr or None))


def bd_decode(model: int, prompt_ptr: int, b: int, P: int, G: int, cfg: bd_decode_cfg, tokens_ptr: int,
              commit_ptr: int, fwd_ptr: int):
    _check(lib.bd_decode(model, prompt_ptr, b, P, G, ctypes.byref(cfg), tokens_ptr, commit_ptr, fwd_ptr))


def bd_decode_static(model: int, prompt_ptr: int, b: int, P: int, G: int, cfg: bd_decode_cfg, tokens_ptr: int,
                     commit_ptr: int, fwd_ptr: int):
    _check(lib.bd_decode_static(model, prompt_ptr, b, P, G, ctypes.byref(cfg), tokens_ptr, commit_ptr,
                                fwd_ptr))


def bd_state_reset(model: int, state: int):
    _check(lib.bd_state_reset(model, state))


def bd_state_steps(state: int) -> int:
    n = ctypes.c_int32(0)
    _check(lib.bd_state_steps(state, ctypes.byref(n)))
    return n.value


def bd_state_stats(model: int, state: int):
    out = (ctypes.c_int64 * len(STAT_NAMES))()
    _check(lib.bd_state_stats(model, state, out, len(STAT_NAMES)))
    return dict(zip(STAT_NAMES, list(out)))


def bd_profile(model: int, enable: bool):
    _check(lib.bd_profile(model, 1 if enable else 0))


def bd_profile_read(model: int):
    ms = (ctypes.c_double * len(PROF_KINDS))()
    n = (ctypes.c_int32 * len(PROF_KINDS))()
    _check(lib.bd_profile_read(model, ms, n))
    return {k: (ms[i], n[i]) for i, k in enumerate(PROF_KINDS)}


def bd_plan_projection(N: int, K: int, rows_cap: int, resid: bool):
    """Tile plan of a bf16 projection: (bm, bn, zmax, workspace floats)."""
    bm, bn, zm = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    wsf = ctypes.c_int64()
    _check(lib.bd_plan_projection(N, K, rows_cap, 1 if resid else 0, ctypes.byref(bm), ctypes.byref(bn),
                                  ctypes.byref(zm), ctypes.byref(wsf)))
    return bm.value, bn.value, zm.value, wsf.value


def bd_kv_pages(n, page_size, max_pages, n_pages, have, want, table, free, free_count, info, rows_cap, row_start, row_seq,
                row_pos, slot, stream=0):
    _check(lib.bd_kv_pages(n, page_size, max_pages, n_pages, have, want, table, free, free_count, info, rows_cap, row_start,
                           row_seq, row_pos, slot, stream))


def bd_kv_store(cache, k, v, dtype, ldk, ldv, n, rows, table, max_pages, row_start, pos0, stream=0):
    _check(lib.bd_kv_store(cache, k, v, dtype, ldk, ldv, n, rows, table, max_pages, row_start, pos0, stream))


def bd_kv_read(cache, k, v, dtype, ldk, ldv, n, rows, table, max_pages, row_start, pos0, stream=0):
    _check(lib.bd_kv_read(cache, k, v, dtype, ldk, ldv, n, rows, table, max_pages, row_start, pos0, stream))


def bd_kv_attention(cache, q, out, dtype, ldq, ldo, n_heads, n, rows, max_rows, table, max_pages, row_start, pos0, kv_len,
                    block_size, scale, ws, ws_bytes, stream=0):
    _check(lib.bd_kv_attention(cache, q, out, dtype, ldq, ldo, n_heads, n, rows, max_rows, table, max_pages, row_start, pos0,
                               kv_len, block_size, scale, ws, ws_bytes, stream))


def bd_kv_attention_workspace(n_heads: int, n_kv_heads: int, head_dim: int, n: int, rows: int, max_rows: int,
                              page_size: int, max_pages: int) -> int:
    out = ctypes.c_int64()
    _check(lib.bd_kv_attention_workspace(n_heads, n_kv_heads, head_dim, n, rows, max_rows, page_size, max_pages,
                                         ctypes.byref(out)))
    return out.value


def bd_token_scores(logits, dtype, ld, logit_rows, vocab, rows, row_index, tokens, suppress, k, logprob, entropy, top_id,
                    top_logprob, ws, ws_bytes, stream=0):
    _check(lib.bd_token_scores(logits, dtype, ld, logit_rows, vocab, rows, row_index, tokens, suppress, k, logprob, entropy,
                               top_id, top_logprob, ws, ws_bytes, stream))


def bd_token_scores_workspace(rows: int, vocab: int, k: int) -> int:
    out = ctypes.c_int64()
    _check(lib.bd_token_scores_workspace(rows, vocab, k, ctypes.byref(out)))
    return out.value


def bd_state_free(state: int):
    _check(lib.bd_state_free(state))


def bd_model_free(model: int):
    _check(lib.bd_model_free(model))


def rl_risk_select(correct, cost, ref_index: int, alpha: float, delta: float):
    """correct: uint8 numpy [m][n]; cost: float64 [m].  Returns
    (V int32[m], p float64[m], valid bool[m], selected, near_ties)."""
    import numpy as np
    c = np.ascontiguousarray(correct, dtype=np.uint8)
    m, n = c.shape
    k = np.ascontiguousarray(cost, dtype=np.float64)
    V = np.zeros(m, dtype=np.int32)
    p = np.zeros(m, dtype=np.float64)
    valid = np.zeros(m, dtype=np.uint8)
    sel = ctypes.c_int32(-1)
    near = ctypes.c_int32(0)
    u8, f64, i32 = ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)
    _check(lib.rl_risk_select(n, m, ref_index, c.ctypes.data_as(u8), k.ctypes.data_as(f64), alpha, delta,
                              V.ctypes.data_as(i32), p.ctypes.data_as(f64), valid.ctypes.data_as(u8),
                              ctypes.byref(sel), ctypes.byref(near)))
    return V, p, valid.astype(bool), sel.value, near.value


_u8, _f64, _i32 = ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)


def _method_order(method: str, order, m: int):
    import numpy as np
    code = RL_METHODS[method]
    o = None if order is None else np.ascontiguousarray(order, dtype=np.int32)
    if o is not None and o.shape != (m,):
        raise ValueError("order must hold m entries")
    return code, o, (None if o is None else o.ctypes.data_as(_i32))


def rl_select(correct, cost, ref_index: int, alpha: float, delta: float, method: str = "holm",
              order=None, mask=None):
    """Returns (V int32[m], p float64[m], valid bool[m], selected)."""
    import numpy as np
    c = np.ascontiguousarray(correct, dtype=np.uint8)
    m, n = c.shape
    k = np.ascontiguousarray(cost, dtype=np.float64)
    code, o, op = _method_order(method, order, m)
    mk = None if mask is None else np.ascontiguousarray(mask, dtype=np.uint8)
    V = np.zeros(m, dtype=np.int32)
    p = np.zeros(m, dtype=np.float64)
    valid = np.zeros(m, dtype=np.uint8)
    sel = ctypes.c_int32(-1)
    _check(lib.rl_select(n, m, ref_index, c.ctypes.data_as(_u8), None if mk is None else mk.ctypes.data_as(_u8),
                         k.ctypes.data_as(_f64), alpha, delta, code, op, V.ctypes.data_as(_i32),
                         p.ctypes.data_as(_f64), valid.ctypes.data_as(_u8), ctypes.byref(sel)))
    return V, p, valid.astype(bool), sel.value


def rl_alpha_sweep(correct, cost, ref_index: int, alphas, delta: float, method: str = "holm", order=None):
    """Returns (selected int32[n_alpha], n_valid int32[n_alpha], alpha_hat or None)."""
    import math
    import numpy as np
    c = np.ascontiguousarray(correct, dtype=np.uint8)
    m, n = c.shape
    k = np.ascontiguousarray(cost, dtype=np.float64)
    a = np.ascontiguousarray(alphas, dtype=np.float64)
    code, o, op = _method_order(method, order, m)
    sel = np.zeros(len(a), dtype=np.int32)
    nval = np.zeros(len(a), dtype=np.int32)
    hat = ctypes.c_double(0.0)
    _check(lib.rl_alpha_sweep(n, m, ref_index, c.ctypes.data_as(_u8), k.ctypes.data_as(_f64),
                              a.ctypes.data_as(_f64), len(a), delta, code, op, sel.ctypes.data_as(_i32),
                              nval.ctypes.data_as(_i32), ctypes.byref(hat)))
    return sel, nval, (None if math.isnan(hat.value) else hat.value)


def rl_split_exceedance(correct, cost, ref_index: int, alpha: float, delta: float, cal_masks,
                        method: str = "holm", order=None):
    """Returns (deployed int32[S], test_violations int32[S], counts int32[4], gain_sum);
    counts = (exceed_test, exceed_pooled, fwer_test, fwer_pooled)."""
    import numpy as np
    c = np.ascontiguousarray(correct, dtype=np.uint8)
    m, n = c.shape
    k = np.ascontiguousarray(cost, dtype=np.float64)
    masks = np.ascontiguousarray(cal_masks, dtype=np.uint8)
    if masks.ndim != 2 or masks.shape[1] != n:
        raise ValueError("cal_masks must be [n_splits][n]")
    S = masks.shape[0]
    code, o, op = _method_order(method, order, m)
    dep = np.zeros(S, dtype=np.int32)
    tv = np.zeros(S, dtype=np.int32)
    counts = np.zeros(4, dtype=np.int32)
    gain = ctypes.c_double(0.0)
    _check(lib.rl_split_exceedance(n, m, ref_index, c.ctypes.data_as(_u8), k.ctypes.data_as(_f64), alpha,
                                   delta, code, op, S, masks.ctypes.data_as(_u8), dep.ctypes.data_as(_i32),
                                   tv.ctypes.data_as(_i32), counts.ctypes.data_as(_i32), ctypes.byref(gain)))
    return dep, tv, counts, gain.value


def rl_monte_carlo(true_risk, alpha: float, delta: float, u, method: str = "holm", order=None):
    """u: float64 [trials][1 or m][n].  Returns (false_trials, valid_counts int32[m])."""
    import numpy as np
    r = np.ascontiguousarray(true_risk, dtype=np.float64)
    m = r.shape[0]
    uu = np.ascontiguousarray(u, dtype=np.float64)
    if uu.ndim != 3:
        raise ValueError("u must be [trials][k][n]")
    trials, kk, n = uu.shape
    code, o, op = _method_order(method, order, m)
    ft = ctypes.c_int32(0)
    counts = np.zeros(m, dtype=np.int32)
    _check(lib.rl_monte_carlo(n, m, r.ctypes.data_as(_f64), alpha, delta, code, op, trials, kk,
                              uu.ctypes.data_as(_f64), ctypes.byref(ft), counts.ctypes.data_as(_i32)))
    return ft.value, counts


# ---------------------------------------------------------------- torch helpers
def model_cfg_from(w) -> bd_model_cfg:
    """Build the C config from a workload description (attribute access)."""
    return bd_model_cfg(n_layers=w.n_layers, d_model=w.d_model, n_heads=w.n_heads, n_kv_heads=w.n_kv_heads,
                        head_dim=w.head_dim, ffn_dim=w.ffn_dim, vocab=w.vocab, n_experts=w.n_experts,
                        top_k=w.top_k, expert_ffn=w.expert_ffn, n_shared=w.n_shared, rms_eps=w.rms_eps,
                        rope_theta=w.rope_theta, logit_scale=w.logit_scale, mask_id=w.vocab - 1,
                        dtype=BD_BF16 if w.dtype == "bf16" else BD_F32)


class Model:
    """Device copy of the weights plus the library handle."""

    def __init__(self, workload, weights, device: str = "cuda:0", wq=None, kv=None, kv_page: int = 32):
        """``wq``: None (weights in the model dtype), "fp8" or "mxfp4"
        (decoder-layer projections quantized by the library, see
        bd_quantize_fp8 and bd_quantize_mxfp4).  ``kv``: None (K and V as bf16
        pairs, or fp32) or "fp8" (8-bit pages of ``kv_page`` tokens, see
        bd_model_kv_cache)."""
        import numpy as np
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.w = workload
        self.tensors = []
        for a in weights:
            a = np.ascontiguousarray(a)
            if a.dtype == np.uint16:
                t = torch.from_numpy(a.view(np.int16)).to(self.device)
            else:
                t = torch.from_numpy(a.astype(np.float32)).to(self.device)
            self.tensors.append(t)
        self.stream = torch.cuda.current_stream(self.device)
        torch.cuda.synchronize(self.device)
        self.cfg = model_cfg_from(workload)
        self.cfg.wq = WQ[wq]
        self.wq = wq
        self.handle = bd_init_model(self.cfg, [t.data_ptr() for t in self.tensors], self.stream.cuda_stream)
        if kv is not None:
            if kv != "fp8":
                self.close()
                raise ValueError(f"unknown cache kind {kv!r}")
            try:
                bd_model_kv_cache(self.handle, BD_KV_FP8, kv_page)
            except BDError:
                self.close()
                raise

    def close(self):
        if self.handle:
            bd_model_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class State:
    """A decode state of ``b`` sequences (prefill done on creation)."""

    def __init__(self, model: Model, prompts, G: int, tau: float, n_inflight: int, block_size: int,
                 tau_semi=None, tau_add: float = 0.0, skip_masked: bool = False):
        torch = model.torch
        self.m = model
        self.prompts = torch.as_tensor(prompts, dtype=torch.int32).to(model.device).contiguous()
        self.b, self.P = self.prompts.shape
        self.G = G
        self.cfg = decode_cfg(tau, n_inflight, block_size, tau_semi, tau_add, skip_masked)
        self.handle = bd_prefill(model.handle, self.prompts.data_ptr(), self.b, self.P, G, self.cfg)

    def step(self, conf=None, tok=None, logits=None):
        ptr = lambda t: 0 if t is None else t.data_ptr()
        bd_denoise_step(self.m.handle, self.handle, ptr(conf), ptr(tok), ptr(logits))

    def commit(self, want_done: bool = False):
        return bd_commit(self.m.handle, self.handle, want_done)

    def read(self):
        torch = self.m.torch
        t = torch.empty((self.b, self.G), dtype=torch.int32, device=self.m.device)
        c = torch.empty((self.b, self.G), dtype=torch.int32, device=self.m.device)
        f = torch.empty((self.b,), dtype=torch.int32, device=self.m.device)
        bd_state_read(self.m.handle, self.handle, t.data_ptr(), c.data_ptr(), f.data_ptr())
        return t.cpu().numpy(), c.cpu().numpy(), f.cpu().numpy()

    def reset(self):
        bd_state_reset(self.m.handle, self.handle)

    @property
    def steps(self) -> int:
        return bd_state_steps(self.handle)

    def stats(self) -> dict:
        return bd_state_stats(self.m.handle, self.handle)

    def close(self):
        if self.handle:
            bd_state_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def decode(model: Model, prompts, G: int, tau: float, n_inflight: int, block_size: int, tau_semi=None,
           tau_add: float = 0.0, skip_masked: bool = False, static: bool = False):
    """Whole decode through ``bd_decode`` (``bd_decode_static`` with
    ``static``); returns numpy (tokens, commit_step, forwards)."""
    torch = model.torch
    pr = torch.as_tensor(prompts, dtype=torch.int32).to(model.device).contiguous()
    b, P = pr.shape
    t = torch.empty((b, G), dtype=torch.int32, device=model.device)
    c = torch.empty((b, G), dtype=torch.int32, device=model.device)
    f = torch.empty((b,), dtype=torch.int32, device=model.device)
    cfg = decode_cfg(tau, n_inflight, block_size, tau_semi, tau_add, skip_masked)
    entry = bd_decode_static if static else bd_decode
    entry(model.handle, pr.data_ptr(), b, P, G, cfg, t.data_ptr(), c.data_ptr(), f.data_ptr())
    return t.cpu().numpy(), c.cpu().numpy(), f.cpu().numpy()


# ---------------------------------------------------------------- paged KV cache, token scores
_loaded_torch = None
_raw_stream = None


def _torch():
    """torch, imported at the first call that takes tensors."""
    global _loaded_torch, _raw_stream
    if _loaded_torch is None:
        import torch
        # the stream's handle without the Stream object around it, 0.1 against 1.9 us a call
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _loaded_torch = torch
    return _loaded_torch


def _ints(t, what: str, shape, device):
    """Checks an int32 tensor of the call's device: contiguous, of ``shape`` (None: any size)."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous torch.int32 tensor on {device}")
    have = t.shape
    if have != shape and (len(have) != len(shape) or any(w is not None and w != g for w, g in zip(shape, have))):
        raise ValueError(f"{what} must have shape {tuple('*' if w is None else w for w in shape)}, got {tuple(have)}")
    return t.data_ptr()


def _rows(t, what: str, heads, hd: int, device, dtype=None):
    """A [rows][heads][hd] tensor whose rows may be strided; returns (pointer, row stride, rows)."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or t.dim() != 3 or t.device != device or t.shape[1:] != (heads, hd):
        raise ValueError(f"{what} must be a [rows][{heads}][{hd}] tensor on {device}")
    have = t.dtype
    if (have is not torch.bfloat16 and have is not torch.float32) or (dtype is not None and have is not dtype):
        raise ValueError(f"{what} must be bfloat16 or float32, as the other rows are")
    ld, head, one = t.stride()
    if one != 1 or (head != hd and heads > 1):
        raise ValueError(f"the heads of a row of {what} must lie side by side")
    n = t.shape[0]
    # a single row's stride is whatever torch says: it is never taken
    return t.data_ptr(), (ld if n > 1 else heads * hd), n


def _run(call, device, *args):
    """``call`` with ``args`` and the current stream of ``device``, which is current meanwhile."""
    if device.type != "cuda":
        raise ValueError("the tensors must be on a GPU")
    cuda = _torch().cuda
    if cuda.current_device() == device.index:
        call(*args, _raw_stream(device.index))
    else:
        with cuda.device(device):
            call(*args, _raw_stream(device.index))


class KVCache:
    """A pool of 8-bit pages (see ``bd_kv_cache`` in bd.h) over the caller's tensors: ``k``, ``v`` uint8
    [pages][kv heads][page_size * head_dim], ``k_scale``, ``v_scale`` float32 [pages][kv heads]."""

    def __init__(self, k, v, k_scale, v_scale, page_size: int):
        torch = _torch()
        if k.dim() != 3 or page_size < 1 or k.shape[2] % page_size:
            raise ValueError("k must be [pages][kv heads][page_size * head_dim]")
        self.device = k.device
        for t, what, like in ((k, "k", k), (v, "v", k), (k_scale, "k_scale", k), (v_scale, "v_scale", k)):
            scale = what.endswith("scale")
            if t.dtype != (torch.float32 if scale else torch.uint8) or t.device != self.device or not t.is_contiguous() or \
                    tuple(t.shape) != tuple(like.shape[:2] if scale else like.shape):
                raise ValueError(f"{what} has the wrong type, device, shape or layout")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_kv_heads = k.shape[0], k.shape[1]
        self.page_size, self.head_dim = page_size, k.shape[2] // page_size
        self.desc = bd_kv_cache(n_pages=self.n_pages, n_kv_heads=self.n_kv_heads, head_dim=self.head_dim,
                                page_size=page_size, k=k.data_ptr(), v=v.data_ptr(), k_scale=k_scale.data_ptr(),
                                v_scale=v_scale.data_ptr())
        self.ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_size: int, device="cuda:0"):
        """A cleared pool."""
        torch = _torch()
        z = lambda: torch.zeros((n_pages, n_kv_heads, page_size * head_dim), dtype=torch.uint8, device=device)
        s = lambda: torch.full((n_pages, n_kv_heads), 2.0 ** -126, dtype=torch.float32, device=device)
        return cls(z(), z(), s(), s(), page_size)


class KVPages:
    """What ``kv_pages`` returns: the new rows' ``row_start``, ``row_seq``, ``row_pos``, ``slot``, and ``info``
    (free pages, rows, pages missing, pages taken) as device tensors."""
    __slots__ = ("row_start", "row_seq", "row_pos", "slot", "info")

    def __init__(self, row_start, row_seq, row_pos, slot, info):
        self.row_start, self.row_seq, self.row_pos, self.slot, self.info = row_start, row_seq, row_pos, slot, info


def kv_pages(have, want, table, free, free_count, page_size: int, rows_cap: int) -> KVPages:
    """Block tables, slot maps and the free list from the requests' held and wanted lengths (``bd_kv_pages``).
    ``table`` [n][max_pages] and ``free`` [pages] change in place; ``free_count`` [1] does not, the new count is
    ``info[0]`` (``info[:1]`` is the next call's ``free_count``)."""
    torch = _torch()
    dev = table.device
    n, max_pages = table.shape
    args = (_ints(have, "have", (n,), dev), _ints(want, "want", (n,), dev), _ints(table, "table", (n, None), dev),
            _ints(free, "free", (None,), dev), _ints(free_count, "free_count", (1,), dev))
    if rows_cap < 0:
        raise ValueError("need rows_cap >= 0")
    i = torch.empty(n + 5 + 2 * rows_cap, dtype=torch.int32, device=dev)
    slot = torch.empty(rows_cap, dtype=torch.int64, device=dev)
    p = i.data_ptr()
    _run(bd_kv_pages, dev, n, page_size, max_pages, free.shape[0], *args, p, rows_cap, p + 16, p + 4 * (n + 5),
         p + 4 * (n + 5 + rows_cap), slot.data_ptr())
    info, row_start, row_seq, row_pos = i.split((4, n + 1, rows_cap, rows_cap))
    return KVPages(row_start, row_seq, row_pos, slot, info)


def _kv_rows(call, cache, table, row_start, pos0, k, v):
    dev = cache.device
    n, max_pages = table.shape
    kp, ldk, rows = _rows(k, "k", cache.n_kv_heads, cache.head_dim, dev)
    vp, ldv, vrows = _rows(v, "v", cache.n_kv_heads, cache.head_dim, dev, k.dtype)
    if vrows != rows:
        raise ValueError("k and v must have the same rows")
    t, rs, p0 = (_ints(table, "table", (n, None), dev), _ints(row_start, "row_start", (n + 1,), dev),
                 _ints(pos0, "pos0", (n,), dev))
    _run(call, dev, cache.ref, kp, vp, BD_F32 if k.dtype is _torch().float32 else BD_BF16, ldk, ldv, n, rows, t, max_pages, rs,
         p0)


def kv_store(cache: KVCache, k, v, table, row_start, pos0):
    """Writes the rows ``k``, ``v`` [rows][kv heads][head_dim] (bfloat16 or float32) into the pages of their
    requests, from position ``pos0[s]`` on (``bd_kv_store``)."""
    _kv_rows(bd_kv_store, cache, table, row_start, pos0, k, v)


def kv_read(cache: KVCache, table, row_start, pos0, k, v):
    """Fills the rows ``k``, ``v`` with the cached values of the tokens from ``pos0[s]`` on (``bd_kv_read``)."""
    _kv_rows(bd_kv_read, cache, table, row_start, pos0, k, v)


def kv_attention(cache: KVCache, q, table, row_start, pos0, kv_len, block_size: int = 1, max_rows: int = 0, scale: float = 0.0,
                 out=None, workspace=None):
    """Block-causal attention of the query rows ``q`` [rows][heads][head_dim] over the pages (``bd_kv_attention``).
    ``workspace``: a uint8 tensor of ``bd_kv_attention_workspace`` bytes; allocated for the call if None."""
    torch = _torch()
    dev = cache.device
    n, max_pages = table.shape
    H = q.shape[1] if q.dim() == 3 else 0
    qp, ldq, rows = _rows(q, "q", H, cache.head_dim, dev)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    op, ldo, orows = _rows(out, "out", H, cache.head_dim, dev, q.dtype)
    if orows != rows:
        raise ValueError("q and out must have the same rows")
    t, rs, p0, kl = (_ints(table, "table", (n, None), dev), _ints(row_start, "row_start", (n + 1,), dev),
                     _ints(pos0, "pos0", (n,), dev), _ints(kv_len, "kv_len", (n,), dev))
    if workspace is None:
        wb = bd_kv_attention_workspace(H, cache.n_kv_heads, cache.head_dim, n, rows, max_rows, cache.page_size, max_pages)
        if wb:
            workspace = torch.empty(wb, dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    else:
        wb = workspace.numel() * workspace.element_size()
    _run(bd_kv_attention, dev, cache.ref, qp, op, BD_F32 if q.dtype is torch.float32 else BD_BF16, ldq, ldo, H, n, rows, max_rows,
         t, max_pages, rs, p0, kl, block_size, scale, workspace.data_ptr() if wb else None, wb)
    return out


class TokenScores:
    """What ``token_scores`` returns: ``logprob`` [rows] (None without tokens), ``entropy`` [rows], ``top_id`` and
    ``top_logprob`` [rows][k]."""
    __slots__ = ("logprob", "entropy", "top_id", "top_logprob")

    def __init__(self, logprob, entropy, top_id, top_logprob):
        self.logprob, self.entropy, self.top_id, self.top_logprob = logprob, entropy, top_id, top_logprob


def token_scores(logits, tokens=None, k: int = 1, suppress: int = -1, row_index=None) -> TokenScores:
    """Log probability of ``tokens`` [rows], entropy and the ``k`` most probable tokens of the rows of ``logits``
    [logit rows][vocab] (bfloat16 or float32, rows may be strided), or of the rows ``row_index`` [rows] names
    (``bd_token_scores``).  ``suppress``: a token left out of the softmax."""
    torch = _torch()
    if logits.dim() != 2 or logits.stride(1) != 1 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be [rows][vocab] of bfloat16 or float32 with adjacent columns")
    dev = logits.device
    R, V = logits.shape
    ip = None if row_index is None else _ints(row_index, "row_index", (None,), dev)
    rows = R if row_index is None else row_index.shape[0]
    tp = None if tokens is None else _ints(tokens, "tokens", (rows,), dev)
    ld = logits.stride(0) if R > 1 else V
    need = bd_token_scores_workspace(rows, V, k) // 4          # whole floats: 16-byte parts
    f = torch.empty(need + rows * (2 + k), dtype=torch.float32, device=dev)
    top_id = torch.empty((rows, k), dtype=torch.int32, device=dev)
    ws = f.data_ptr()
    p = ws + 4 * need
    _run(bd_token_scores, dev, logits.data_ptr(), BD_F32 if logits.dtype is torch.float32 else BD_BF16, ld, R, V, rows, ip, tp,
         suppress, k, p if tokens is not None else None, p + 4 * rows, top_id.data_ptr(), p + 8 * rows, ws if need else None,
         4 * need)
    _, logprob, entropy, top_logprob = f.split((need, rows, rows, rows * k))
    return TokenScores(None if tokens is None else logprob, entropy, top_id, top_logprob.view(rows, k))
