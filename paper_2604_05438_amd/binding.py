"""ctypes binding of libtkphi with the same entry-point names as include/tkphi.h.

Argument marshalling only: every step of the path runs in the library's HIP kernels.
torch is used for device memory and streams (tensor.data_ptr(), current stream).
The shared library is loaded on first use; if it has not been built the call raises
(there is no CPU fallback).
"""
from __future__ import annotations

import ctypes as C
import os
import threading

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtkphi.so")

TKPHI_OK = 0
TKPHI_EINVAL, TKPHI_ESHAPE, TKPHI_EALIGN, TKPHI_EWORKSPACE, TKPHI_EHIP, TKPHI_EUNSUPPORTED = -1, -2, -3, -4, -5, -6
TKPHI_F32, TKPHI_BF16 = 0, 1
TKPHI_MODE_SUB, TKPHI_MODE_NOSUB, TKPHI_MODE_TOPK_ONLY = 0, 1, 2
TKPHI_FLAG_DIAG = 0x100
TKPHI_PHI_EXP_AFFINE, TKPHI_PHI_MLP = 0, 1
TKPHI_DIAG_STRIDE = 8
TKPHI_DEV_BAD_LENGTH, TKPHI_DEV_CLAMPED, TKPHI_DEV_BAD_PAGE = 1, 2, 4

EXPORTS = (
    "tkphi_workspace_bytes", "tkphi_build_summaries", "tkphi_decode", "tkphi_decode_static", "tkphi_decode_stage_times",
    "tkphi_check_problems",
    "tkphi_read_device_status", "tkphi_budget_paper", "tkphi_budget_mid", "tkphi_status_string",
    "tkphi_last_error",
    "tkphi_paged_workspace_bytes", "tkphi_kv_append", "tkphi_paged_attention", "tkphi_block_attention",
)


def aux_stride(d_head: int) -> int:
    return 4 + 2 * d_head


class tkphi_tuning(C.Structure):
    _fields_ = [
        ("force_generic", C.c_int32), ("scan_chunk", C.c_int32), ("interleave", C.c_int32),
        ("build_chunk", C.c_int32), ("mlp_block", C.c_int32), ("mlp_mode", C.c_int32),
        ("select_mode", C.c_int32), ("select_test", C.c_int32),
        ("reserved", C.c_int32 * 4),
    ]


MLP_MODES = {"": 0, "chain": 0, "blocks": 1, "unfused": 2}


class tkphi_config(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("d_phi", C.c_int32),
        ("n_sink", C.c_int32), ("n_tail", C.c_int32), ("kv_dtype", C.c_int32),
        ("score_scale", C.c_float), ("phi_in_scale", C.c_float), ("phi_norm_coef", C.c_float),
        ("cache_features", C.c_int32), ("phi_kind", C.c_int32), ("d_emb", C.c_int32), ("max_gen", C.c_int32),
        ("tuning", tkphi_tuning),
    ]


class tkphi_mlp(C.Structure):
    _fields_ = [
        ("Ws", C.c_void_p), ("bs", C.c_void_p), ("W1", C.c_void_p), ("b1", C.c_void_p),
        ("W2", C.c_void_p), ("b2", C.c_void_p), ("Wo", C.c_void_p), ("bo", C.c_void_p),
        ("alpha", C.c_float), ("reserved", C.c_int32),
    ]


class tkphi_problem(C.Structure):
    _fields_ = [
        ("K", C.c_void_p), ("V", C.c_void_p), ("stride_head", C.c_int64), ("stride_tok", C.c_int64),
        ("Wq", C.c_void_p), ("bq", C.c_void_p), ("Wk", C.c_void_p), ("bk", C.c_void_p),
        ("S", C.c_void_p), ("u", C.c_void_p), ("q", C.c_void_p), ("out", C.c_void_p),
        ("topk_idx", C.c_void_p), ("aux", C.c_void_p), ("scores", C.c_void_p), ("diag", C.c_void_p), ("phi_cache", C.c_void_p),
        ("mlp_q", C.c_void_p), ("mlp_k", C.c_void_p),
        ("L", C.c_int32), ("topk", C.c_int32), ("n_gen", C.c_int32), ("reserved", C.c_int32),
    ]


class tkphi_paged_config(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("kv_dtype", C.c_int32),
        ("score_scale", C.c_float), ("page_tokens", C.c_int32),
        ("stride_page", C.c_int64), ("stride_head", C.c_int64), ("stride_tok", C.c_int64),
        ("window", C.c_int32), ("rot_dim", C.c_int32), ("rot_adjacent", C.c_int32), ("block", C.c_int32),
        ("first_blocks", C.c_int32), ("last_blocks", C.c_int32), ("top_blocks", C.c_int32), ("workgroups", C.c_int32),
        ("reserved", C.c_int32 * 4),
    ]


class tkphi_step(C.Structure):
    _fields_ = [
        ("seqs", C.c_void_p), ("pages", C.c_void_p), ("n_seqs", C.c_int32), ("max_pages", C.c_int32), ("rows", C.c_int32),
        ("max_new", C.c_int32), ("max_len", C.c_int32), ("reserved", C.c_int32),
    ]


class tkphi_kv_pool(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("M", C.c_void_p), ("n_pages", C.c_int32), ("reserved", C.c_int32)]


class tkphi_new_rows(C.Structure):
    heads, angles = "kv_q_heads", 1 << 30          # (make_new_rows: which note of the config the heads have to match, elements of inv_freq)
    _fields_ = [
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_rot", C.c_void_p), ("inv_freq", C.c_void_p),
        ("q_row", C.c_int64), ("q_head", C.c_int64), ("k_row", C.c_int64), ("k_head", C.c_int64),
        ("v_row", C.c_int64), ("v_head", C.c_int64), ("q_rot_row", C.c_int64), ("q_rot_head", C.c_int64),
    ]


class tkphi_attention_rows(C.Structure):
    _fields_ = [
        ("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
        ("q_row", C.c_int64), ("q_head", C.c_int64), ("out_row", C.c_int64), ("out_head", C.c_int64),
    ]


_lib = None
_lock = threading.Lock()


def lib() -> C.CDLL:
    """Loads libtkphi.so (once).  Raises if it is missing: build it with
    `python -m paper_2604_05438_amd.build`."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not built; run `python -m paper_2604_05438_amd.build`")
        L = C.CDLL(LIB_PATH)
        cfgp, probp = C.POINTER(tkphi_config), C.c_void_p
        L.tkphi_workspace_bytes.restype = C.c_size_t
        L.tkphi_workspace_bytes.argtypes = [cfgp, C.c_int32, C.c_int32, C.c_int32]
        L.tkphi_build_summaries.restype = C.c_int
        L.tkphi_build_summaries.argtypes = [cfgp, probp, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.tkphi_decode.restype = C.c_int
        L.tkphi_decode.argtypes = [cfgp, probp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                   C.c_size_t, C.c_void_p]
        L.tkphi_decode_static.restype = C.c_int
        L.tkphi_decode_static.argtypes = [cfgp, probp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        L.tkphi_decode_stage_times.restype = C.c_int
        L.tkphi_decode_stage_times.argtypes = [cfgp, probp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                               C.c_size_t, C.c_void_p, C.POINTER(C.c_float)]
        L.tkphi_check_problems.restype = C.c_int
        L.tkphi_check_problems.argtypes = [cfgp, C.POINTER(tkphi_problem), C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        L.tkphi_read_device_status.restype = C.c_int
        L.tkphi_read_device_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_uint32)]
        L.tkphi_budget_paper.restype = C.c_int32
        L.tkphi_budget_paper.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32]
        L.tkphi_budget_mid.restype = C.c_int32
        L.tkphi_budget_mid.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32]
        L.tkphi_status_string.restype = C.c_char_p
        L.tkphi_status_string.argtypes = [C.c_int32]
        L.tkphi_last_error.restype = C.c_char_p
        L.tkphi_last_error.argtypes = []
        pcfg, stepp, poolp = C.POINTER(tkphi_paged_config), C.POINTER(tkphi_step), C.POINTER(tkphi_kv_pool)
        L.tkphi_paged_workspace_bytes.restype = C.c_size_t
        L.tkphi_paged_workspace_bytes.argtypes = [pcfg, stepp]
        for name, rows in (("tkphi_kv_append", tkphi_new_rows), ("tkphi_paged_attention", tkphi_attention_rows),
                           ("tkphi_block_attention", tkphi_attention_rows)):
            f = getattr(L, name)
            f.restype = C.c_int
            f.argtypes = [pcfg, stepp, poolp, C.POINTER(rows), C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
        return L


class TkphiError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        super().__init__(f"tkphi status {status} ({tkphi_status_string(status)}): {detail}")


def _check(status: int) -> None:
    if status != TKPHI_OK:
        raise TkphiError(status, tkphi_last_error())


# ---- entry points (same names as the C ABI) ---------------------------------------------
def tkphi_status_string(status: int) -> str:
    return lib().tkphi_status_string(status).decode()


def tkphi_last_error() -> str:
    return lib().tkphi_last_error().decode()


def tkphi_budget_paper(L: int, r_bp: int, n_sink: int, n_tail: int) -> int:
    return lib().tkphi_budget_paper(L, r_bp, n_sink, n_tail)


def tkphi_budget_mid(L: int, r_bp: int, n_sink: int, n_tail: int) -> int:
    return lib().tkphi_budget_mid(L, r_bp, n_sink, n_tail)


def tkphi_workspace_bytes(cfg: tkphi_config, n_problems: int, max_L: int, max_K: int) -> int:
    return lib().tkphi_workspace_bytes(C.byref(cfg), n_problems, max_L, max_K)


def tkphi_check_problems(cfg: tkphi_config, problems_host, n_problems: int, max_L: int, max_K: int,
                         for_decode: bool) -> None:
    _check(lib().tkphi_check_problems(C.byref(cfg), problems_host, n_problems, max_L, max_K, int(for_decode)))


def tkphi_build_summaries(cfg: tkphi_config, problems_dev_ptr: int, n_problems: int, max_L: int,
                          workspace_ptr: int, workspace_bytes: int, stream: int) -> None:
    _check(lib().tkphi_build_summaries(C.byref(cfg), problems_dev_ptr, n_problems, max_L, workspace_ptr,
                                       workspace_bytes, stream))


def tkphi_decode(cfg: tkphi_config, problems_dev_ptr: int, n_problems: int, max_L: int, max_K: int,
                 mode: int, workspace_ptr: int, workspace_bytes: int, stream: int) -> None:
    _check(lib().tkphi_decode(C.byref(cfg), problems_dev_ptr, n_problems, max_L, max_K, mode, workspace_ptr,
                              workspace_bytes, stream))


def tkphi_decode_static(cfg: tkphi_config, problems_dev_ptr: int, n_problems: int, max_L: int, max_K: int,
                        mode: int, stream: int) -> None:
    _check(lib().tkphi_decode_static(C.byref(cfg), problems_dev_ptr, n_problems, max_L, max_K, mode, stream))


STATIC_SCRATCH_BYTES = 32 << 20


STAGES = ("score_mid", "select_plan", "select_emit", "select_resolve", "gather", "merge", "phi_q", "prep", "select")
SELECT_SPILL, SELECT_FILTERED = 1, 2          # tkphi_tuning::select_mode


def tkphi_decode_stage_times(cfg: tkphi_config, problems_dev_ptr: int, n_problems: int, max_L: int, max_K: int,
                             mode: int, workspace_ptr: int, workspace_bytes: int, stream: int) -> list:
    out = (C.c_float * len(STAGES))()
    _check(lib().tkphi_decode_stage_times(C.byref(cfg), problems_dev_ptr, n_problems, max_L, max_K, mode,
                                          workspace_ptr, workspace_bytes, stream, out))
    return list(out)


def tkphi_read_device_status(workspace_ptr: int, stream: int) -> int:
    out = C.c_uint32(0)
    _check(lib().tkphi_read_device_status(workspace_ptr, stream, C.byref(out)))
    return out.value


def tkphi_paged_workspace_bytes(cfg: tkphi_paged_config, step: tkphi_step) -> int:
    return lib().tkphi_paged_workspace_bytes(C.byref(cfg), C.byref(step))


def _fits(cfg, step, pool, io, heads) -> None:
    """The tensors that cfg, step, pool and io were made from (make_step and so on) against each other: the kernels go by the config's types, heads and
    strides and by the step's rows.  heads: the note of the config that the rows' heads have to match.  (A struct filled by hand has
    no notes: nothing is compared then.  0.3 us where all is well.)"""
    try:
        (rows, form, device), want, has, geometry, on, at = io.form, getattr(cfg, heads), pool.form, cfg.pool, pool.device, step.device
    except AttributeError:
        return
    if rows >= step.rows and form == want and has == geometry and on == device == at >= 0 and (pool.blocks == cfg.blocks or not (pool.blocks and cfg.blocks)):
        return
    if rows < step.rows:
        raise ValueError(f"{rows} rows for a step of {step.rows}")
    if form != want:
        raise ValueError(f"rows of (storage type, channels, heads) {form} for a config of {want}")
    if not on == device == at >= 0:
        raise ValueError(f"rows, pool and step on GPUs {device}, {on}, {at} (-1: not on a GPU)")
    if pool.blocks != cfg.blocks and pool.blocks and cfg.blocks:
        raise ValueError(f"M has {pool.blocks} blocks per page, the config {cfg.blocks}")
    for name, a, b in zip(("storage type", "channels", "KV heads", "tokens per page", "stride of pages", "stride of heads", "stride of tokens"), has, geometry):
        if a != b and a is not None and b is not None:
            raise ValueError(f"pool: {name} {a}, in the config {b}")


def tkphi_kv_append(cfg: tkphi_paged_config, step: tkphi_step, pool: tkphi_kv_pool, io: tkphi_new_rows, workspace_ptr: int,
                    workspace_bytes: int, stream: int) -> None:
    _fits(cfg, step, pool, io, io.heads)
    if 2 * io.angles < cfg.rot_dim:
        raise ValueError(f"inv_freq has {io.angles} elements for rot_dim = {cfg.rot_dim}")
    _check(lib().tkphi_kv_append(cfg, step, pool, io, workspace_ptr, workspace_bytes, stream))


def tkphi_paged_attention(cfg: tkphi_paged_config, step: tkphi_step, pool: tkphi_kv_pool, io: tkphi_attention_rows, workspace_ptr: int,
                          workspace_bytes: int, stream: int) -> None:
    _fits(cfg, step, pool, io, "q_heads")
    _check(lib().tkphi_paged_attention(cfg, step, pool, io, workspace_ptr, workspace_bytes, stream))


def tkphi_block_attention(cfg: tkphi_paged_config, step: tkphi_step, pool: tkphi_kv_pool, io: tkphi_attention_rows, workspace_ptr: int,
                          workspace_bytes: int, stream: int) -> None:
    _fits(cfg, step, pool, io, "q_heads")
    _check(lib().tkphi_block_attention(cfg, step, pool, io, workspace_ptr, workspace_bytes, stream))


# ---- marshalling helpers (device memory via torch) -----------------------------------------
def make_config(n_q_heads, n_kv_heads, d_head, d_phi, n_sink, n_tail, dtype, score_scale, phi_in_scale,
                phi_norm_coef, cache_features=0, phi_kind=0, d_emb=0, max_gen=0, tuning=None) -> tkphi_config:
    """tuning: optional dict of tkphi_tuning fields (launch-geometry overrides; omitted fields stay 0 = default)."""
    kv = {"bf16": TKPHI_BF16, "f32": TKPHI_F32}[dtype] if isinstance(dtype, str) else int(dtype)
    cfg = tkphi_config(n_q_heads, n_kv_heads, d_head, d_phi, n_sink, n_tail, kv, score_scale, phi_in_scale,
                       phi_norm_coef, int(cache_features), int(phi_kind), int(d_emb), int(max_gen))
    for name, value in (tuning or {}).items():
        setattr(cfg.tuning, name, int(value))
    return cfg


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def make_problem(K, V, Wq, bq, Wk, bk, S, u, q=None, out=None, topk_idx=None, aux=None, scores=None,
                 L=None, topk=0, diag=None, phi_cache=None, mlp_q=None, mlp_k=None, n_gen=0) -> tkphi_problem:
    """Fills a tkphi_problem from torch device tensors (K, V: [Hkv][L + n_gen][d], last dim contiguous)."""
    assert K.stride(-1) == 1 and V.stride(-1) == 1 and K.stride() == V.stride()
    return tkphi_problem(
        _ptr(K), _ptr(V), K.stride(0), K.stride(1), _ptr(Wq), _ptr(bq), _ptr(Wk), _ptr(bk), _ptr(S), _ptr(u),
        _ptr(q), _ptr(out), _ptr(topk_idx), _ptr(aux), _ptr(scores), _ptr(diag), _ptr(phi_cache), _ptr(mlp_q), _ptr(mlp_k),
        int(K.shape[1] - n_gen if L is None else L), int(topk), int(n_gen), 0)


def upload_mlp(maps: dict, device="cuda"):
    """One side ("q" or "k") of inputs.make_mlp_phi, already on the device as torch tensors ->
    (device uint8 tensor holding the tkphi_mlp array [H], list of tensors to keep alive)."""
    import torch
    H = maps["alpha"].shape[0]
    arr = (tkphi_mlp * H)()
    for h in range(H):
        arr[h] = tkphi_mlp(_ptr(maps["Ws"][h]), _ptr(maps["bs"][h]), _ptr(maps["W1"][h]), _ptr(maps["b1"][h]),
                           _ptr(maps["W2"][h]), _ptr(maps["b2"][h]), _ptr(maps["Wo"][h]), _ptr(maps["bo"][h]),
                           float(maps["alpha"][h]), 0)
    raw = bytes(memoryview(arr).cast("B"))
    return torch.frombuffer(bytearray(raw), dtype=torch.uint8).to(device)


def upload_problems(problems, device="cuda"):
    """Host list of tkphi_problem -> (host ctypes array, device uint8 tensor holding the table)."""
    import torch
    arr = (tkphi_problem * len(problems))(*problems)
    raw = bytes(memoryview(arr).cast("B"))
    host = torch.frombuffer(bytearray(raw), dtype=torch.uint8)
    return arr, host.to(device)


def alloc_workspace(nbytes: int, device="cuda"):
    import torch
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


# ---- the paged cache -----------------------------------------------------------------------
# The structs hold addresses only: the caller keeps the tensors.  What the calls compare with the config (_fits) is noted beside the fields.
def _tensor(name, t, dims, dtype=None, adjoin=True):
    if t.dim() != dims or (adjoin and t.shape[-1] > 1 and t.stride(-1) != 1) or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, strides {t.stride()}, {t.dtype}; needs {dims} dimensions"
                         + (", the last one contiguous" if adjoin else "") + (f", {dtype}" if dtype is not None else ""))
    return t


def _storage_type(kv_dtype):
    import torch
    return {TKPHI_BF16: torch.bfloat16, TKPHI_F32: torch.float32}[kv_dtype]


def _kv_dtype(t):
    import torch
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{t.dtype} is no storage type (torch.bfloat16 or torch.float32)")
    return TKPHI_BF16 if t.dtype == torch.bfloat16 else TKPHI_F32


def _pool_form(K):
    """Storage type, channels, heads, tokens and strides; a stride over one element does not matter (None)."""
    return (_kv_dtype(K), K.shape[3], K.shape[1], K.shape[2], *(K.stride(i) if K.shape[i] > 1 else None for i in range(3)))


def _one_device(**tensors):
    """The GPU that all of them are on, -1 for the CPU"""
    devices = {n: t.get_device() for n, t in tensors.items() if t is not None}
    if len(set(devices.values())) > 1:
        raise ValueError(f"tensors on several GPUs (-1: not on one): {devices}")
    return next(iter(devices.values()))


def make_paged_config(n_q_heads, n_kv_heads, d_head, dtype, score_scale, K, V, window=0, rot_dim=0, rot_adjacent=False, block=0,
                      first_blocks=0, last_blocks=0, top_blocks=0, workgroups=0) -> tkphi_paged_config:
    """K, V: the pool's tensors as [pages][KV heads][tokens per page][channels], in any memory order with adjoining channels and
    the same strides."""
    kv = {"bf16": TKPHI_BF16, "f32": TKPHI_F32}[dtype] if isinstance(dtype, str) else int(dtype)
    for name, t in (("K", K), ("V", V)):
        _tensor(name, t, 4, _storage_type(kv))
        if t.shape != K.shape or t.stride() != K.stride() or t.shape[1] != n_kv_heads or t.shape[3] != d_head:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, strides {t.stride()} do not fit K and the heads")
    cfg = tkphi_paged_config(int(n_q_heads), int(n_kv_heads), int(d_head), kv, float(score_scale), K.shape[2], K.stride(0), K.stride(1),
                             K.stride(2), int(window), int(rot_dim), int(bool(rot_adjacent)), int(block), int(first_blocks), int(last_blocks),
                             int(top_blocks), int(workgroups))
    cfg.pool, cfg.blocks = _pool_form(K), K.shape[2] // cfg.block if cfg.block > 0 else 0
    cfg.q_heads, cfg.kv_heads, cfg.kv_q_heads = (kv, cfg.d_head, cfg.n_q_heads), (kv, cfg.d_head, cfg.n_kv_heads), (kv, cfg.d_head, cfg.n_kv_heads, cfg.n_q_heads)
    return cfg


def make_step(seqs, pages, rows: int, max_new: int, max_len: int) -> tkphi_step:
    """seqs: int32 [n][4] (cached, new tokens, first row, 0); pages: int32 [n][max_pages], both contiguous on the device."""
    import torch
    for name, t in (("seqs", seqs), ("pages", pages)):
        _tensor(name, t, 2, torch.int32)
        if not t.is_contiguous() or t.shape[0] != seqs.shape[0]:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, strides {t.stride()}; one contiguous row per sequence")
    if seqs.shape[1] != 4:
        raise ValueError("seqs: four words per sequence")
    step = tkphi_step(_ptr(seqs), _ptr(pages), seqs.shape[0], pages.shape[1], int(rows), int(max_new), int(max_len), 0)
    step.device = _one_device(seqs=seqs, pages=pages)
    return step


def make_pool(K, V, M=None) -> tkphi_kv_pool:
    """K, V as for make_paged_config; M: mean keys [pages][KV heads][blocks per page][channels], contiguous, or None."""
    for name, t in (("K", K), ("V", V)):
        _tensor(name, t, 4, K.dtype)
        if t.shape != K.shape or t.stride() != K.stride():
            raise ValueError(f"{name}: shape {tuple(t.shape)}, strides {t.stride()} are not those of K")
    if M is not None:
        _tensor("M", M, 4, K.dtype)
        if not M.is_contiguous() or M.shape[:2] != K.shape[:2] or M.shape[3] != K.shape[3]:
            raise ValueError(f"M: shape {tuple(M.shape)}, strides {M.stride()} do not fit K")
    pool = tkphi_kv_pool(_ptr(K), _ptr(V), _ptr(M), K.shape[0], 0)
    pool.form, pool.blocks, pool.device = _pool_form(K), 0 if M is None else M.shape[2], _one_device(K=K, V=V, M=M)
    return pool


def make_new_rows(q, k, v, q_rot, inv_freq=None) -> tkphi_new_rows:
    """[rows][heads][channels]; q and q_rot may both be None.  inv_freq: float64."""
    import torch
    st = []
    for name, t in (("q", q), ("k", k), ("v", v), ("q_rot", q_rot)):
        if t is None and name in ("q", "q_rot"):
            st += [0, 0]
            continue
        _tensor(name, t, 3, k.dtype)
        if t.shape[0] != k.shape[0] or t.shape[2] != k.shape[2] or (name == "v" and t.shape != k.shape) or (name == "q_rot" and t.shape != q.shape):
            raise ValueError(f"{name}: shape {tuple(t.shape)} does not fit k {tuple(k.shape)}")
        st += [t.stride(0), t.stride(1)]
    if inv_freq is not None:
        _tensor("inv_freq", inv_freq, 1, torch.float64)
    io = tkphi_new_rows(_ptr(q), _ptr(k), _ptr(v), _ptr(q_rot), _ptr(inv_freq), *st)
    io.form = (k.shape[0], (_kv_dtype(k), k.shape[2], k.shape[1]) + (() if q is None else (q.shape[1],)), _one_device(k=k, v=v, q=q, q_rot=q_rot, inv_freq=inv_freq))
    if q is None:
        io.heads = "kv_heads"
    if inv_freq is not None:
        io.angles = inv_freq.shape[0]
    return io


def make_attention_rows(q, out, lse=None) -> tkphi_attention_rows:
    """q, out: [rows][query heads][channels]; lse: contiguous float32 [rows][query heads] or None."""
    import torch
    _tensor("q", q, 3)
    _tensor("out", out, 3, q.dtype)
    if out.shape != q.shape:
        raise ValueError(f"out: shape {tuple(out.shape)} does not fit q {tuple(q.shape)}")
    if lse is not None:
        _tensor("lse", lse, 2, torch.float32)
        if not lse.is_contiguous() or lse.shape != q.shape[:2]:
            raise ValueError(f"lse: shape {tuple(lse.shape)}, strides {lse.stride()} do not fit q")
    io = tkphi_attention_rows(_ptr(q), _ptr(out), _ptr(lse), q.stride(0), q.stride(1), out.stride(0), out.stride(1))
    io.form = (q.shape[0], (_kv_dtype(q), q.shape[2], q.shape[1]), _one_device(q=q, out=out, lse=lse))
    return io


def alloc_paged_workspace(nbytes: int, device="cuda"):
    """A zeroed workspace, which the calls on the paged cache ask for (they leave it fit for the next call)."""
    import torch
    return torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=device)


def current_stream_ptr() -> int:
    import torch
    if torch.cuda.is_initialized() and hasattr(torch._C, "_cuda_getCurrentRawStream"):
        # the same handle without a torch.cuda.Stream object around it: 0.3 instead of 2.8 us per call
        return int(torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()))
    return int(torch.cuda.current_stream().cuda_stream)
