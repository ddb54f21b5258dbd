"""Thin binding of libdifr.so, the B200 token-scoring library.

The functions carry the names of the C entry points in include/difr.h and only
marshal arguments: torch supplies device memory and streams, every step of the
scoring path runs in the library's CUDA kernels.  There is no CPU fallback: a
missing or unloadable library raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libdifr.so")

DIFR_OK = 0
STATUS_NAMES = {0: "DIFR_OK", -1: "DIFR_ERR_INVALID_ARG", -2: "DIFR_ERR_SHAPE", -3: "DIFR_ERR_ALIGN",
                -4: "DIFR_ERR_WORKSPACE", -5: "DIFR_ERR_CUDA", -6: "DIFR_ERR_ARCH", -7: "DIFR_ERR_TIMEOUT"}

EXPORTS = ("difr_workspace_bytes", "difr_filtered_workspace_bytes", "difr_score_gm", "difr_score_ipt",
           "difr_score_both", "difr_score_gm_filtered", "difr_score_ipt_filtered", "difr_score_gm_static",
           "difr_admissible", "difr_exfiltratable_bits", "difr_detect", "difr_expand_seeds", "difr_logits", "difr_philox",
           "difr_mx_codes_bytes", "difr_mx_scales_bytes", "difr_mx_quantize", "difr_mx_dequantize", "difr_rms_norm",
           "difr_mx_logits", "difr_block_norm", "difr_verify_workspace_bytes", "difr_verify_drafts",
           "difr_w4_codes_bytes", "difr_w4_scales_bytes", "difr_w4_quantize", "difr_w4_dequantize", "difr_w4_workspace_bytes",
           "difr_w4_logits",
           "difr_selftest_wait", "difr_selftest_mx_wait", "difr_selftest_w4_wait",
           "difr_debug_plan_override", "difr_status_string", "difr_version")
STATIC_SCRATCH_BYTES = 16 << 20  # DIFR_STATIC_SCRATCH_BYTES
DIFR_BF16, DIFR_F16, DIFR_F32 = 0, 1, 2
DIFR_MX8, DIFR_MX4 = 8, 4


class DifrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


class _COut(ctypes.Structure):
    _fields_ = [
        ("sigma", ctypes.c_float), ("eps", ctypes.c_float),
        ("score", ctypes.c_void_p), ("margin", ctypes.c_void_p), ("argmax", ctypes.c_void_p),
        ("runner_up", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("p_claimed", ctypes.c_void_p),
        ("cdf_lo", ctypes.c_void_p), ("u", ctypes.c_void_p), ("row_status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("device_status", ctypes.c_void_p),
        ("event_fused_start", ctypes.c_void_p), ("event_fused_stop", ctypes.c_void_p),
        ("rank", ctypes.c_void_p), ("y_max", ctypes.c_void_p), ("y_second", ctypes.c_void_p),
        ("sigma_ipt", ctypes.c_float), ("score_ipt", ctypes.c_void_p), ("cutoff", ctypes.c_void_p),
        ("temperatures", ctypes.c_void_p),
    ]


class _CFilter(ctypes.Structure):
    _fields_ = [("top_k", ctypes.c_int32), ("top_p", ctypes.c_float), ("s", ctypes.c_int32),
                ("top_k_rows", ctypes.c_void_p), ("top_p_rows", ctypes.c_void_p),
                ("min_p", ctypes.c_float), ("min_p_rows", ctypes.c_void_p), ("any_size", ctypes.c_int32)]


class _CNormOut(ctypes.Structure):
    _fields_ = [("residual", ctypes.c_void_p), ("ld_residual", ctypes.c_int64), ("h", ctypes.c_void_p),
                ("ldh", ctypes.c_int64), ("mx_format", ctypes.c_int32), ("codes", ctypes.c_void_p),
                ("scales", ctypes.c_void_p)]


class _CBlock(ctypes.Structure):
    _fields_ = [("post_weight", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("ld_gate", ctypes.c_int64),
                ("post_eps", ctypes.c_float), ("scale", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("weight_offset", ctypes.c_float)]


class _CDrafts(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("max_drafts", ctypes.c_int32),
                ("draft_probs", ctypes.c_void_p), ("ld_draft", ctypes.c_int64), ("draft_tokens", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p), ("accept_words", ctypes.c_void_p), ("sample_words", ctypes.c_void_p),
                ("temperature", ctypes.c_float), ("temperatures", ctypes.c_void_p)]


class _CDraftsOut(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("n_accepted", ctypes.c_void_p), ("p_draft", ctypes.c_void_p),
                ("status", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads csrc/libdifr.so (built by paper_2511_02620_b200.build.build())."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2511_02620_b200.build` "
                              "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        L.difr_workspace_bytes.restype = ctypes.c_size_t
        L.difr_workspace_bytes.argtypes = [ctypes.c_int64] * 3
        score_args = [ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_int64] * 3 + [ctypes.POINTER(_COut),
                                                                                      ctypes.c_void_p]
        for name in ("difr_score_gm", "difr_score_ipt", "difr_score_both", "difr_score_gm_static"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = score_args
        L.difr_detect.restype = ctypes.c_int
        L.difr_detect.argtypes = [ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                  ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_void_p]
        L.difr_filtered_workspace_bytes.restype = ctypes.c_size_t
        L.difr_filtered_workspace_bytes.argtypes = [ctypes.c_int64] * 3
        for name in ("difr_score_gm_filtered", "difr_score_ipt_filtered"):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = ([ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_int64] * 3
                                         + [ctypes.POINTER(_CFilter), ctypes.POINTER(_COut), ctypes.c_void_p])
        L.difr_admissible.restype = ctypes.c_int
        L.difr_admissible.argtypes = ([ctypes.c_void_p] * 4 + [ctypes.c_float] + [ctypes.c_int64] * 3
                                      + [ctypes.c_void_p] * 4 + [ctypes.c_float] * 2
                                      + [ctypes.POINTER(ctypes.c_float), ctypes.c_int32, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                         ctypes.c_void_p])
        L.difr_exfiltratable_bits.restype = ctypes.c_int
        L.difr_exfiltratable_bits.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                              ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                              ctypes.c_void_p, ctypes.c_void_p]
        L.difr_expand_seeds.restype = ctypes.c_int
        L.difr_expand_seeds.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                        ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
        L.difr_logits.restype = ctypes.c_int
        L.difr_logits.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.difr_philox.restype = ctypes.c_int
        L.difr_philox.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
        L.difr_selftest_wait.restype = ctypes.c_int
        L.difr_selftest_wait.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]
        L.difr_debug_plan_override.restype = ctypes.c_int
        L.difr_debug_plan_override.argtypes = [ctypes.c_int32] * 3
        L.difr_status_string.restype = ctypes.c_char_p
        L.difr_status_string.argtypes = [ctypes.c_int]
        L.difr_version.restype = ctypes.c_int
        v, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.difr_mx_codes_bytes.restype = ctypes.c_size_t
        L.difr_mx_codes_bytes.argtypes = [i32, i64, i64]
        L.difr_mx_scales_bytes.restype = ctypes.c_size_t
        L.difr_mx_scales_bytes.argtypes = [i64, i64]
        L.difr_mx_quantize.restype = ctypes.c_int
        L.difr_mx_quantize.argtypes = [v, i32, i64, i64, i64, i32, v, v, v]
        L.difr_mx_dequantize.restype = ctypes.c_int
        L.difr_mx_dequantize.argtypes = [v, v, i32, i64, i64, v, i32, i64, v]
        L.difr_rms_norm.restype = ctypes.c_int
        L.difr_rms_norm.argtypes = [v, i64, v, i64, v, i32, i64, i64, ctypes.c_float, ctypes.POINTER(_CNormOut), v]
        L.difr_mx_logits.restype = ctypes.c_int
        L.difr_mx_logits.argtypes = [v, v, v, v, i32, i64, i64, i64, v, i32, i64, v, v]
        L.difr_block_norm.restype = ctypes.c_int
        L.difr_block_norm.argtypes = [v, i64, v, i64, ctypes.POINTER(_CBlock), v, i32, i64, i64, ctypes.c_float,
                                      ctypes.POINTER(_CNormOut), v]
        L.difr_w4_codes_bytes.restype = ctypes.c_size_t
        L.difr_w4_codes_bytes.argtypes = [i64, i64]
        L.difr_w4_scales_bytes.restype = ctypes.c_size_t
        L.difr_w4_scales_bytes.argtypes = [i64, i64, i32]
        L.difr_w4_workspace_bytes.restype = ctypes.c_size_t
        L.difr_w4_workspace_bytes.argtypes = [i64, i64]
        L.difr_w4_quantize.restype = ctypes.c_int
        L.difr_w4_quantize.argtypes = [v, i32, i64, i64, i64, i32, v, v, v]
        L.difr_w4_dequantize.restype = ctypes.c_int
        L.difr_w4_dequantize.argtypes = [v, v, i32, i64, i64, v, i32, i64, v]
        L.difr_w4_logits.restype = ctypes.c_int
        L.difr_w4_logits.argtypes = [v, i64, v, v, i32, i64, i64, i64, v, i32, i64, v, ctypes.c_size_t, v, v]
        L.difr_verify_workspace_bytes.restype = ctypes.c_size_t
        L.difr_verify_workspace_bytes.argtypes = [i64, i64, i64]
        L.difr_verify_drafts.restype = ctypes.c_int
        L.difr_verify_drafts.argtypes = [ctypes.POINTER(_CDrafts), i64, i64, i64, ctypes.POINTER(_CDraftsOut), v]
        L.difr_selftest_mx_wait.restype = ctypes.c_int
        L.difr_selftest_mx_wait.argtypes = [i32, i64, i64, i64, v, i32, i64, i32, i64, v, v]
        L.difr_selftest_w4_wait.restype = ctypes.c_int
        L.difr_selftest_w4_wait.argtypes = [i64, i64, i64, v, i32, i64, i32, i64, v, v]
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch

    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(t, dtype, shape, name):
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor")
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise TypeError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def difr_workspace_bytes(T: int, d: int, V: int) -> int:
    return int(lib().difr_workspace_bytes(T, d, V))


def difr_version() -> int:
    return int(lib().difr_version())


def difr_status_string(status: int) -> str:
    return lib().difr_status_string(status).decode()


@dataclass
class DifrOut:
    """Estimator parameters and output tensors of a scoring call (mirrors `difr_out`)."""
    sigma: float
    eps: float
    score: "object"
    margin: "object" = None
    argmax: "object" = None
    runner_up: "object" = None
    lse: "object" = None
    p_claimed: "object" = None
    cdf_lo: "object" = None
    u: "object" = None
    row_status: "object" = None
    workspace: "object" = None
    device_status: "object" = None
    event_fused_start: int = 0  # raw cudaEvent_t handles (0: none)
    event_fused_stop: int = 0
    rank: "object" = None       # int32 [T]: ask for the raw-logit rank of the claimed token (GM calls)
    y_max: "object" = None      # float [T]: largest / second largest l + Temp*G (GM calls); difr_admissible needs them
    y_second: "object" = None
    sigma_ipt: float = 0.0      # difr_score_both: width of the IPT estimator
    score_ipt: "object" = None  # difr_score_both: float [T]
    cutoff: "object" = None     # difr_score_gm_filtered: float [T], the filter's cutoff per row
    temperatures: "object" = None  # float [T]: one temperature per row instead of the call's scalar

    @staticmethod
    def allocate(T: int, d: int, V: int, sigma: float, eps: float = 1e-12, device="cuda"):
        import torch

        f = lambda: torch.empty(T, dtype=torch.float32, device=device)
        i = lambda: torch.empty(T, dtype=torch.int32, device=device)
        nbytes = max(difr_workspace_bytes(T, d, V), 16)
        return DifrOut(sigma, eps, f(), f(), i(), i(), f(), f(), f(), f(), i(),
                       torch.empty(nbytes, dtype=torch.uint8, device=device),
                       torch.zeros(1, dtype=torch.int32, device=device))

    def _c(self) -> _COut:
        ws = self.workspace
        return _COut(float(self.sigma), float(self.eps), _ptr(self.score), _ptr(self.margin), _ptr(self.argmax),
                     _ptr(self.runner_up), _ptr(self.lse), _ptr(self.p_claimed), _ptr(self.cdf_lo), _ptr(self.u),
                     _ptr(self.row_status), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                     _ptr(self.device_status), ctypes.c_void_p(self.event_fused_start or None),
                     ctypes.c_void_p(self.event_fused_stop or None), _ptr(self.rank), _ptr(self.y_max),
                     _ptr(self.y_second), float(self.sigma_ipt), _ptr(self.score_ipt), _ptr(self.cutoff),
                     _ptr(self.temperatures))


def _score(fn_name, h, W, tokens, seeds, positions, temperature, out: DifrOut, stream):
    import torch

    T, d = h.shape
    V = W.shape[0]
    _check(h, torch.bfloat16, (T, d), "h")
    _check(W, torch.bfloat16, (V, d), "W")
    _check(tokens, torch.int32, (T,), "tokens")
    _check(seeds, torch.int64, (T,), "seeds")  # uint64 bit patterns carried in int64 storage
    _check(positions, torch.int32, (T,), "positions")  # uint32 bit patterns
    c = out._c()
    rc = getattr(lib(), fn_name)(_ptr(h), _ptr(W), _ptr(tokens), _ptr(seeds), _ptr(positions), float(temperature),
                                 T, d, V, ctypes.byref(c), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, fn_name)
    return out


def difr_score_gm(h, W, tokens, seeds, positions, temperature, out: DifrOut, stream=None) -> DifrOut:
    """Token-DiFR (Gumbel-max) scores; see include/difr.h."""
    return _score("difr_score_gm", h, W, tokens, seeds, positions, temperature, out, stream)


def difr_score_ipt(h, W, tokens, seeds, positions, temperature, out: DifrOut, stream=None) -> DifrOut:
    """Token-IPT-DiFR scores; see include/difr.h."""
    return _score("difr_score_ipt", h, W, tokens, seeds, positions, temperature, out, stream)


def difr_score_both(h, W, tokens, seeds, positions, temperature, out: DifrOut, stream=None) -> DifrOut:
    """Token-DiFR and Token-IPT-DiFR scores from one pass (`out.sigma_ipt`, `out.score_ipt`); see include/difr.h."""
    return _score("difr_score_both", h, W, tokens, seeds, positions, temperature, out, stream)


def difr_filtered_workspace_bytes(T: int, d: int, V: int) -> int:
    return int(lib().difr_filtered_workspace_bytes(T, d, V))


def difr_score_ipt_filtered(h, W, tokens, seeds, positions, temperature, top_k, top_p, out: DifrOut, stream=None,
                            min_p=0.0, any_size=False):
    """Token-IPT-DiFR on the filtered distribution; workspace as for difr_score_gm_filtered."""
    return difr_score_gm_filtered(h, W, tokens, seeds, positions, temperature, top_k, top_p, 1, out, stream,
                                  _fn="difr_score_ipt_filtered", min_p=min_p, any_size=any_size)


def difr_score_gm_filtered(h, W, tokens, seeds, positions, temperature, top_k, top_p, s, out: DifrOut, stream=None,
                           _fn="difr_score_gm_filtered", min_p=0.0, any_size=False):
    """Alg. Token-DiFR in full: top-k / top-p cutoff, B_i terms, s competitors; `out.workspace` must hold
    difr_filtered_workspace_bytes(T, d, V) bytes.  `top_k` (int32) and `top_p` (float32) may be device tensors
    of T values, one per row (`min_p` likewise), and `out.temperatures` one temperature per row; `any_size`
    lets such per-row values go beyond 128 kept ids.
    See include/difr.h."""
    import torch

    T, d = h.shape
    V = W.shape[0]
    _check(h, torch.bfloat16, (T, d), "h")
    _check(W, torch.bfloat16, (V, d), "W")
    _check(tokens, torch.int32, (T,), "tokens")
    _check(seeds, torch.int64, (T,), "seeds")
    _check(positions, torch.int32, (T,), "positions")
    c = out._c()
    k_rows = top_k if isinstance(top_k, torch.Tensor) else None
    p_rows = top_p if isinstance(top_p, torch.Tensor) else None
    if k_rows is not None:
        _check(k_rows, torch.int32, (T,), "top_k")
    if p_rows is not None:
        _check(p_rows, torch.float32, (T,), "top_p")
    m_rows = min_p if isinstance(min_p, torch.Tensor) else None
    if m_rows is not None:
        _check(m_rows, torch.float32, (T,), "min_p")
    f = _CFilter(0 if k_rows is not None else int(top_k), 1.0 if p_rows is not None else float(top_p), int(s),
                 _ptr(k_rows), _ptr(p_rows), 0.0 if m_rows is not None else float(min_p), _ptr(m_rows),
                 1 if any_size else 0)
    rc = getattr(lib(), _fn)(_ptr(h), _ptr(W), _ptr(tokens), _ptr(seeds), _ptr(positions),
                             float(temperature), T, d, V, ctypes.byref(f), ctypes.byref(c), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, _fn)
    return out


def difr_admissible(h, W, seeds, positions, temperature, scored: DifrOut, taus, counts, row_status=None, stream=None):
    """Admissible-set sizes |A_t(tau)| for up to four thresholds; `scored` holds argmax, runner_up, y_max, y_second,
    sigma, eps and the workspace of a difr_score_gm call on the same inputs; `counts` is int32 [len(taus), T];
    `row_status` (uint32 bits in an int32 [T] tensor, optional) receives bit 5 for rows whose list overflowed."""
    import torch

    T, d = h.shape
    V = W.shape[0]
    taus = [float(t) for t in taus]
    _check(counts, torch.int32, (len(taus), T), "counts")
    arr = (ctypes.c_float * len(taus))(*taus)
    ws = scored.workspace
    rc = lib().difr_admissible(_ptr(h), _ptr(W), _ptr(seeds), _ptr(positions), float(temperature), T, d, V,
                               _ptr(scored.argmax), _ptr(scored.runner_up), _ptr(scored.y_max), _ptr(scored.y_second),
                               float(scored.sigma), float(scored.eps), arr, len(taus), _ptr(counts), _ptr(row_status),
                               _ptr(ws), ws.numel() * ws.element_size(), _ptr(scored.device_status), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_admissible")
    return counts


def difr_exfiltratable_bits(classes, counts, rank_cutoff, V, seq_offsets=None, bits=None, seq_bits=None, stream=None):
    """Per-token / per-sequence information bound from the risk classes and admissible-set sizes."""
    T = classes.shape[0]
    n_seq = 1 if seq_offsets is None else seq_offsets.shape[0] - 1
    rc = lib().difr_exfiltratable_bits(_ptr(classes), _ptr(counts), int(rank_cutoff), int(V), _ptr(seq_offsets), n_seq,
                                       T, _ptr(bits), _ptr(seq_bits), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_exfiltratable_bits")
    return bits, seq_bits


def difr_expand_seeds(seeds, tokens, seq_offsets=None, prompt_hashes=None, expanded=None, stream=None):
    """Sequential randomness expansion: per-row seeds (int64 tensor holding the uint64 words) that also depend
    on the prompt hash of the row's sequence and on the claimed tokens before it.  `expanded` may be `seeds`."""
    T = seeds.shape[0]
    n_seq = 1 if seq_offsets is None else seq_offsets.shape[0] - 1
    if expanded is None:
        import torch
        expanded = torch.empty_like(seeds)
    rc = lib().difr_expand_seeds(_ptr(seeds), _ptr(tokens), _ptr(seq_offsets), n_seq, _ptr(prompt_hashes), T,
                                 _ptr(expanded), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_expand_seeds")
    return expanded


def difr_score_gm_static(h, W, tokens, seeds, positions, temperature, out: DifrOut, stream=None) -> DifrOut:
    """difr_score_gm for callers that cannot allocate scratch memory: `out.workspace` is ignored (it may be
    None) and the library's built-in 16 MiB array is used instead.  Raises DifrError(DIFR_ERR_WORKSPACE) for
    problems that need more.  Calls on one device share that array, so do not let two of them overlap."""
    return _score("difr_score_gm_static", h, W, tokens, seeds, positions, temperature, out, stream)


def difr_detect(scores, threshold, margins=None, ranks=None, rank_cutoff=0, seq_offsets=None, flags=None,
                seq_stats=None, stream=None):
    """Threshold flags and per-sequence statistics; `seq_stats` is an int32 [n_seq, 4] tensor whose rows are
    (n_flagged, n_match, bits of float sum, bits of float min)."""
    T = scores.shape[0]
    n_seq = 1 if seq_offsets is None else seq_offsets.shape[0] - 1
    rc = lib().difr_detect(_ptr(scores), float(threshold), _ptr(margins), _ptr(ranks), int(rank_cutoff),
                           _ptr(seq_offsets), n_seq, T, _ptr(flags), _ptr(seq_stats), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_detect")
    return flags, seq_stats


def difr_logits(h, W, logits, device_status=None, stream=None):
    T, d = h.shape
    V = W.shape[0]
    rc = lib().difr_logits(_ptr(h), _ptr(W), T, d, V, _ptr(logits), _ptr(device_status), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_logits")
    return logits


def difr_selftest_wait(status2, limit_cycles, stream=None):
    """Runs the bounded-wait self-test; `status2` is an int32 [2] CUDA tensor."""
    rc = lib().difr_selftest_wait(_ptr(status2), int(limit_cycles), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_selftest_wait")
    return status2


def difr_debug_plan_override(strips: int = 0, group: int = 0, l2_mb: int = 0) -> None:
    """Validation aid: fixes the planner's strip count / raster group / L2 share for later calls (0: its own)."""
    rc = lib().difr_debug_plan_override(int(strips), int(group), int(l2_mb))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_debug_plan_override")


def difr_philox(ctr, key, out, stream=None):
    rc = lib().difr_philox(_ptr(ctr), _ptr(key), ctr.shape[0], _ptr(out), _stream(stream))
    if rc != DIFR_OK:
        raise DifrError(rc, "difr_philox")
    return out


# ------------------------------------------------- around the LM head: the final norm, heads in 8 or 4 bits
def difr_mx_codes_bytes(format: int, rows: int, d: int) -> int:
    return int(lib().difr_mx_codes_bytes(format, rows, d))


def difr_mx_scales_bytes(rows: int, d: int) -> int:
    return int(lib().difr_mx_scales_bytes(rows, d))


@dataclass(slots=True)
class MxTensor:
    """A microscaled tensor of `rows` x `d` values (layout in include/difr.h)."""
    codes: "object"   # uint8 [rows, pitch bytes]
    scales: "object"  # uint8 [difr_mx_scales_bytes(rows, d)]
    format: int       # DIFR_MX8 or DIFR_MX4
    rows: int
    d: int

    @staticmethod
    def allocate(rows: int, d: int, format: int, device="cuda"):
        import torch

        if rows > 0 and difr_mx_codes_bytes(format, rows, d) == 0:
            raise ValueError(f"no microscaled tensor of {rows} x {d} values in format {format}")
        # (the bytes of rows behind the last are nobody's: zeros, so that two equal tensors have equal buffers)
        return MxTensor(torch.empty(rows, (d + 31) // 32 * 4 * format, dtype=torch.uint8, device=device),
                        torch.zeros(difr_mx_scales_bytes(rows, d), dtype=torch.uint8, device=device), format, rows, d)


@dataclass(slots=True)
class NormOut:
    """Output tensors of difr_rms_norm (mirrors `difr_norm_out`); None: not wanted."""
    h: "object" = None         # bf16 [T, d]
    residual: "object" = None  # [T, d] of x's type
    mx: MxTensor = None


_torch = None  # the module, once a call has needed it (an import statement costs each call a quarter of a microsecond)
_DTYPES = {}   # torch dtype -> difr_dtype
_ANY_DTYPE, _WIDE_DTYPE = (DIFR_BF16, DIFR_F16, DIFR_F32), (DIFR_BF16, DIFR_F32)


def _load_torch():
    global _torch
    import torch

    _DTYPES.update({torch.bfloat16: DIFR_BF16, torch.float16: DIFR_F16, torch.float32: DIFR_F32})
    _torch = torch


def _matrix(t, name, dtypes, shape=None, device=None):
    """A CUDA matrix whose rows are contiguous; returns (C dtype, row stride, device index)."""
    if _torch is None:
        _load_torch()
    try:
        index = t.get_device()
        code = _DTYPES.get(t.dtype)
        rows, cols = t.shape
        ld, step = t.stride()
    except (AttributeError, ValueError):
        raise TypeError(f"{name} must be a CUDA matrix") from None
    if index < 0:
        raise TypeError(f"{name} must be a CUDA matrix")
    if code not in dtypes:
        raise TypeError(f"{name}: {t.dtype} is not supported here")
    if shape is not None and (rows, cols) != shape:
        raise TypeError(f"{name}: expected {tuple(shape)}, got {(rows, cols)}")
    if device is not None and index != device:
        raise TypeError(f"{name} is on device {index}, not on {device}")
    if rows <= 1 and ld < cols:
        ld = cols
    if (step != 1 and cols > 1) or ld < cols:
        raise TypeError(f"{name}: the rows must be contiguous and must not overlap")
    return code, ld, index


def _check_mx(mx, name, device):
    if not isinstance(mx, MxTensor) or mx.format not in (DIFR_MX8, DIFR_MX4):
        raise TypeError(f"{name} must be an MxTensor of 8 or 4 bits")
    rows, d = mx.rows, mx.d
    _check_bytes(mx.codes, rows * ((d + 31) // 32 * 4 * mx.format), name, "codes", device)
    _check_bytes(mx.scales, (rows + 127) // 128 * ((d + 127) // 128) * 512, name, "scales", device)


def _check_bytes(t, n, name, what, device):
    if not isinstance(t, _torch.Tensor) or t.dtype != _torch.uint8 or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{name}.{what} must be {n} contiguous bytes (uint8)")
    if t.get_device() != device:
        raise TypeError(f"{name}.{what} is on {t.device}, not on CUDA device {device}")


def _call(name, device, stream, *args):
    """Calls an entry point with device number `device` current, on the given stream or that device's current one."""
    if stream is None:
        # (the handle alone: building a torch.cuda.Stream costs 2 us a call)
        raw = _torch._C._cuda_getCurrentRawStream(device)
    elif stream.device.index != device:
        raise TypeError(f"the stream is on {stream.device}, the tensors on CUDA device {device}")
    else:
        raw = stream.cuda_stream
    fn = getattr(_lib or lib(), name)
    if _torch._C._cuda_getDevice() == device:
        rc = fn(*args, raw)
    else:
        with _torch.cuda.device(device):
            rc = fn(*args, raw)
    if rc != DIFR_OK:
        raise DifrError(rc, name)


def difr_mx_quantize(x, out: MxTensor, stream=None) -> MxTensor:
    """Microscaled codes and scales of a matrix (bf16, fp16 or fp32); see include/difr.h."""
    dtype, ld, device = _matrix(x, "x", _ANY_DTYPE)
    _check_mx(out, "out", device)
    if (out.rows, out.d) != x.shape:
        raise TypeError(f"out is {out.rows} x {out.d}, x {tuple(x.shape)}")
    _call("difr_mx_quantize", device, stream, x.data_ptr(), dtype, out.rows, out.d, ld, out.format,
          out.codes.data_ptr(), out.scales.data_ptr())
    return out


def difr_mx_dequantize(mx: MxTensor, out, stream=None):
    """The values of a microscaled tensor, as bf16 (what the scoring calls take) or fp32."""
    dtype, ld, device = _matrix(out, "out", _WIDE_DTYPE)
    _check_mx(mx, "mx", device)
    if (mx.rows, mx.d) != out.shape:
        raise TypeError(f"out is {tuple(out.shape)}, the tensor {mx.rows} x {mx.d}")
    _call("difr_mx_dequantize", device, stream, mx.codes.data_ptr(), mx.scales.data_ptr(), mx.format, mx.rows, mx.d,
          out.data_ptr(), dtype, ld)
    return out


def difr_rms_norm(x, weight, eps, out: NormOut, residual=None, stream=None) -> NormOut:
    """Final root-mean-square norm of x (+ residual); `out.h` feeds the scoring calls, `out.mx` difr_mx_logits."""
    dtype, ldx, device = _matrix(x, "x", _ANY_DTYPE)
    shape = x.shape
    _check_weight(weight, "weight", x, device)
    residual_p, ldr = None, 0
    if residual is not None:
        ldr = _matrix(residual, "residual", (dtype,), shape, device)[1]
        residual_p = residual.data_ptr()
    _call("difr_rms_norm", device, stream, x.data_ptr(), ldx, residual_p, ldr, weight.data_ptr(), dtype, shape[0],
          shape[1], eps, ctypes.byref(_norm_out(out, shape, dtype, device)))
    return out


def _check_weight(weight, name, x, device):
    if (not isinstance(weight, _torch.Tensor) or weight.dtype != x.dtype or weight.get_device() != device
            or weight.dim() != 1 or weight.numel() != x.shape[1] or not weight.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous {x.dtype} [{x.shape[1]}] on {x.device}")


def _norm_out(out, shape, dtype, device):
    stream_p = h_p = codes_p = scales_p = None
    ld_stream = ldh = fmt = 0
    if out.residual is not None:
        ld_stream = _matrix(out.residual, "out.residual", (dtype,), shape, device)[1]
        stream_p = out.residual.data_ptr()
    if out.h is not None:
        ldh = _matrix(out.h, "out.h", (DIFR_BF16,), shape, device)[1]
        h_p = out.h.data_ptr()
    mx = out.mx
    if mx is not None:
        _check_mx(mx, "out.mx", device)
        if (mx.rows, mx.d) != shape:
            raise TypeError(f"out.mx is {mx.rows} x {mx.d}, x {tuple(shape)}")
        fmt, codes_p, scales_p = mx.format, mx.codes.data_ptr(), mx.scales.data_ptr()
    return _CNormOut(stream_p, ld_stream, h_p, ldh, fmt, codes_p, scales_p)


def _check_status_word(t, device):
    if t is not None:
        _check(t, _torch.int32, (1,), "device_status")
        if t.get_device() != device:
            raise TypeError(f"device_status is on {t.device}, not on CUDA device {device}")


def difr_mx_logits(h: MxTensor, W: MxTensor, logits, device_status=None, stream=None):
    """Logits [T, V] (fp32 or bf16) of microscaled hidden states and LM head, both of one format.  A device-side wait that
    runs out leaves NaN where logits were not computed, and DIFR_ERR_TIMEOUT in `device_status` (int32 [1], optional)."""
    dtype, ld, device = _matrix(logits, "logits", _WIDE_DTYPE)
    _check_mx(h, "h", device)
    _check_mx(W, "W", device)
    if h.format != W.format or h.d != W.d:
        raise TypeError(f"h has {h.d} values of {h.format} bits per row, W {W.d} of {W.format}")
    if logits.shape != (h.rows, W.rows):
        raise TypeError(f"logits: expected {(h.rows, W.rows)}, got {tuple(logits.shape)}")
    _check_status_word(device_status, device)
    _call("difr_mx_logits", device, stream, h.codes.data_ptr(), h.scales.data_ptr(), W.codes.data_ptr(),
          W.scales.data_ptr(), h.format, h.rows, h.d, W.rows, logits.data_ptr(), dtype, ld,
          None if device_status is None else device_status.data_ptr())
    return logits


def difr_selftest_mx_wait(format: int, d: int, logits, done_tiles: int, limit_cycles: int, device_status=None, stream=None):
    """How difr_mx_logits ends where a wait runs out: NaN beyond the first `done_tiles` tiles of every pair of CTAs and
    DIFR_ERR_TIMEOUT in `device_status`; see include/difr.h."""
    dtype, ld, device = _matrix(logits, "logits", _WIDE_DTYPE)
    _check_status_word(device_status, device)
    _call("difr_selftest_mx_wait", device, stream, format, logits.shape[0], d, logits.shape[1], logits.data_ptr(), dtype,
          ld, done_tiles, limit_cycles, None if device_status is None else device_status.data_ptr())
    return logits


# ---------------- a decoding step: block norm, 4-bit weights with group scales, verification of drafted tokens
def difr_block_norm(x, residual, weight, eps, out: NormOut, post_weight=None, post_eps=None, gate=None, scale=1.0,
                    residual_scale=1.0, weight_offset=0.0, stream=None) -> NormOut:
    """Norms before and after a block, with its gate ([T, d], or [1, d] for all tokens) and residual scale: the stream
    residual_scale * residual + scale * gate * norm(x) to `out.residual`, its norm to `out.h` / `out.mx`.  Without
    `post_weight` x is taken as it is; `post_eps` None: `eps`; `weight` None: the stream alone.  See include/difr.h."""
    dtype, ldx, device = _matrix(x, "x", _ANY_DTYPE)
    shape = x.shape
    ldr = _matrix(residual, "residual", (dtype,), shape, device)[1]
    weight_p = post_p = gate_p = None
    ld_gate = 0
    if weight is not None:
        _check_weight(weight, "weight", x, device)
        weight_p = weight.data_ptr()
    if post_weight is not None:
        _check_weight(post_weight, "post_weight", x, device)
        post_p = post_weight.data_ptr()
    if gate is not None:
        rows = gate.shape[0] if isinstance(gate, _torch.Tensor) and gate.dim() == 2 else -1
        ld_gate = _matrix(gate, "gate", (dtype,), (1 if rows == 1 else shape[0], shape[1]), device)[1]
        gate_p = gate.data_ptr()
        if rows == 1:
            ld_gate = 0
    block = _CBlock(post_p, gate_p, ld_gate, eps if post_eps is None else post_eps, scale, residual_scale, weight_offset)
    _call("difr_block_norm", device, stream, x.data_ptr(), ldx, residual.data_ptr(), ldr, ctypes.byref(block), weight_p,
          dtype, shape[0], shape[1], eps, ctypes.byref(_norm_out(out, shape, dtype, device)))
    return out


def difr_w4_codes_bytes(rows: int, d: int) -> int:
    return int(lib().difr_w4_codes_bytes(rows, d))


def difr_w4_scales_bytes(rows: int, d: int, group: int) -> int:
    return int(lib().difr_w4_scales_bytes(rows, d, group))


def difr_w4_workspace_bytes(T: int, d: int) -> int:
    return int(lib().difr_w4_workspace_bytes(T, d))


@dataclass(slots=True)
class W4Tensor:
    """A tensor of `rows` x `d` 4-bit integers with group scales (layout in include/difr.h)."""
    codes: "object"   # uint8 [rows, 16 ceil(d / 32)]
    scales: "object"  # bf16 [rows, 8 ceil(groups / 8)]
    group: int        # 32, 64 or 128
    rows: int
    d: int

    @staticmethod
    def allocate(rows: int, d: int, group: int, device="cuda"):
        import torch

        if group not in (32, 64, 128) or (rows > 0 and difr_w4_codes_bytes(rows, d) == 0):
            raise ValueError(f"no 4-bit tensor of {rows} x {d} values in groups of {group}")
        return W4Tensor(torch.empty(rows, (d + 31) // 32 * 16, dtype=torch.uint8, device=device),
                        torch.empty(rows, _w4_scale_pitch(d, group), dtype=torch.bfloat16, device=device), group, rows, d)


def _w4_scale_pitch(d, group):
    return ((d + group - 1) // group + 7) // 8 * 8


def _check_w4(w, name, device):
    if not isinstance(w, W4Tensor) or w.group not in (32, 64, 128):
        raise TypeError(f"{name} must be a W4Tensor in groups of 32, 64 or 128")
    _check_bytes(w.codes, w.rows * ((w.d + 31) // 32 * 16), name, "codes", device)
    s, n = w.scales, w.rows * _w4_scale_pitch(w.d, w.group)
    if not isinstance(s, _torch.Tensor) or s.dtype != _torch.bfloat16 or s.numel() != n or not s.is_contiguous():
        raise TypeError(f"{name}.scales must be {n} contiguous values of bf16")
    if s.get_device() != device:
        raise TypeError(f"{name}.scales is on {s.device}, not on CUDA device {device}")


def difr_w4_quantize(x, out: W4Tensor, stream=None) -> W4Tensor:
    """4-bit codes and group scales of a matrix (bf16, fp16 or fp32); see include/difr.h."""
    dtype, ld, device = _matrix(x, "x", _ANY_DTYPE)
    _check_w4(out, "out", device)
    if (out.rows, out.d) != x.shape:
        raise TypeError(f"out is {out.rows} x {out.d}, x {tuple(x.shape)}")
    _call("difr_w4_quantize", device, stream, x.data_ptr(), dtype, out.rows, out.d, ld, out.group, out.codes.data_ptr(),
          out.scales.data_ptr())
    return out


def difr_w4_dequantize(w: W4Tensor, out, stream=None):
    """The values of a 4-bit tensor, as fp32 (exact) or bf16 (rounded)."""
    dtype, ld, device = _matrix(out, "out", _WIDE_DTYPE)
    _check_w4(w, "w", device)
    if (w.rows, w.d) != out.shape:
        raise TypeError(f"out is {tuple(out.shape)}, the tensor {w.rows} x {w.d}")
    _call("difr_w4_dequantize", device, stream, w.codes.data_ptr(), w.scales.data_ptr(), w.group, w.rows, w.d, out.data_ptr(),
          dtype, ld)
    return out


def difr_w4_logits(h, W: W4Tensor, logits, workspace, device_status=None, stream=None):
    """Logits [T, V] (fp32 or bf16) of bf16 hidden states and a head of 4-bit integers with group scales; `workspace` is a
    uint8 tensor of difr_w4_workspace_bytes(T, d) bytes."""
    dtype, ld, device = _matrix(logits, "logits", _WIDE_DTYPE)
    ldh = _matrix(h, "h", (DIFR_BF16,), None, device)[1]
    _check_w4(W, "W", device)
    T, d = h.shape
    if W.d != d:
        raise TypeError(f"h has {d} values per row, W {W.d}")
    if logits.shape != (T, W.rows):
        raise TypeError(f"logits: expected {(T, W.rows)}, got {tuple(logits.shape)}")
    _check_status_word(device_status, device)
    if (not isinstance(workspace, _torch.Tensor) or workspace.dtype != _torch.uint8 or not workspace.is_contiguous()
            or workspace.get_device() != device):
        raise TypeError(f"workspace must be contiguous bytes (uint8) on CUDA device {device}")
    _call("difr_w4_logits", device, stream, h.data_ptr(), ldh, W.codes.data_ptr(), W.scales.data_ptr(), W.group, T, d, W.rows,
          logits.data_ptr(), dtype, ld, workspace.data_ptr(), workspace.numel(),
          None if device_status is None else device_status.data_ptr())
    return logits


def difr_selftest_w4_wait(d: int, logits, done_tiles: int, limit_cycles: int, device_status=None, stream=None):
    """Validation aid: difr_w4_logits' way out where a wait runs out, without a product; see include/difr.h."""
    dtype, ld, device = _matrix(logits, "logits", _WIDE_DTYPE)
    _check_status_word(device_status, device)
    _call("difr_selftest_w4_wait", device, stream, logits.shape[0], d, logits.shape[1], logits.data_ptr(), dtype, ld, done_tiles,
          limit_cycles, None if device_status is None else device_status.data_ptr())
    return logits


def difr_verify_workspace_bytes(B: int, n_drafts: int, V: int) -> int:
    return int(lib().difr_verify_workspace_bytes(B, n_drafts, V))


@dataclass(slots=True)
class DraftOut:
    """Output tensors and workspace of difr_verify_drafts (mirrors `difr_drafts_out`); p_draft and status may be None."""
    tokens: "object"      # int32 [B, max_drafts + 1]: accepted drafts, the next token, -1 in the rest
    n_accepted: "object"  # int32 [B]
    p_draft: "object"     # float [n_drafts]: the target's probability of every drafted token, NaN where there is none
    status: "object"      # int32 [B] (uint32 bits)
    workspace: "object"   # uint8 [difr_verify_workspace_bytes(B, n_drafts, V)]

    @staticmethod
    def allocate(B: int, n_drafts: int, max_drafts: int, V: int, device="cuda"):
        import torch

        i = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=device)
        return DraftOut(i(B, max_drafts + 1), i(B), torch.empty(n_drafts, dtype=torch.float32, device=device), i(B),
                        torch.empty(difr_verify_workspace_bytes(B, n_drafts, V), dtype=torch.uint8, device=device))


def _vector(t, name, dtype, n, device):
    """Address of a contiguous CUDA vector of n elements."""
    if not isinstance(t, _torch.Tensor) or t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} [{n}]")
    if t.get_device() != device:
        raise TypeError(f"{name} is on {t.device}, not on CUDA device {device}")
    return t.data_ptr()


def difr_verify_drafts(logits, draft_tokens, offsets, accept_words, sample_words, temperature, out: DraftOut,
                       draft_probs=None, stream=None) -> DraftOut:
    """Accepts or refuses drafted tokens against the target's logits [n_drafts + B, V] from given random words (uint32 bits
    in int32 tensors) and samples each request's next token; `temperature` is a number or a float tensor [B].  Request b
    has drafts offsets[b] .. offsets[b + 1] and rows offsets[b] + b ..; see include/difr.h."""
    dtype, ld, device = _matrix(logits, "logits", _ANY_DTYPE)
    rows, V = logits.shape
    i32 = _torch.int32
    B, D = sample_words.shape[0], draft_tokens.shape[0]
    if rows != D + B:
        raise TypeError(f"logits: expected {D} + {B} rows, got {rows}")
    probs_p, ld_probs = None, 0
    if draft_probs is not None:
        ld_probs = _matrix(draft_probs, "draft_probs", (DIFR_F32,), (D, V), device)[1]
        probs_p = draft_probs.data_ptr()
    temps_p = None
    if isinstance(temperature, _torch.Tensor):
        temps_p = _vector(temperature, "temperature", _torch.float32, B, device)
        temperature = 0.0
    tokens, ws = out.tokens, out.workspace
    if (not isinstance(tokens, _torch.Tensor) or tokens.dtype != i32 or tokens.dim() != 2 or tokens.shape[0] != B
            or tokens.shape[1] < 1 or not tokens.is_contiguous() or tokens.get_device() != device):
        raise TypeError(f"out.tokens must be a contiguous int32 [{B}, max_drafts + 1] on CUDA device {device}")
    if not isinstance(ws, _torch.Tensor) or ws.dtype != _torch.uint8 or not ws.is_contiguous() or ws.get_device() != device:
        raise TypeError(f"out.workspace must be contiguous bytes (uint8) on CUDA device {device}")
    c = _CDrafts(logits.data_ptr(), ld, dtype, tokens.shape[1] - 1, probs_p, ld_probs,
                 _vector(draft_tokens, "draft_tokens", i32, D, device), _vector(offsets, "offsets", i32, B + 1, device),
                 _vector(accept_words, "accept_words", i32, D, device),
                 _vector(sample_words, "sample_words", i32, B, device), temperature, temps_p)
    o = _CDraftsOut(tokens.data_ptr(), _vector(out.n_accepted, "out.n_accepted", i32, B, device),
                    None if out.p_draft is None else _vector(out.p_draft, "out.p_draft", _torch.float32, D, device),
                    None if out.status is None else _vector(out.status, "out.status", i32, B, device), ws.data_ptr(), ws.numel())
    _call("difr_verify_drafts", device, stream, ctypes.byref(c), B, D, V, ctypes.byref(o))
    return out
