"""Thin Python binding of libkvec (argument marshalling only).

Every computation runs in the HIP library; this module converts torch tensors
to pointers, strides and the current HIP stream.  There is no CPU fallback: if
libkvec.so is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass, fields

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libkvec.so")
BIND_PATH = os.path.join(HERE, "_kvec_bind.so")

KVEC_OK, KVEC_ERR_INVALID, KVEC_ERR_UNSUPPORTED, KVEC_ERR_WORKSPACE, KVEC_ERR_DEVICE = range(5)
KVEC_BF16, KVEC_F32 = 0, 1
KVEC_HEADS_STD, KVEC_HEADS_ENTROPY = 0, 1
KVEC_Q8_INT8, KVEC_Q8_E4M3 = 0, 1


class KvecError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


class kvec_config(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_layers", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("seq_len", ctypes.c_int32),
        ("window", ctypes.c_int32), ("window_ext", ctypes.c_int32),
        ("budget", ctypes.c_int32), ("pool_kernel", ctypes.c_int32),
        ("n_adjust_heads", ctypes.c_int32),
        ("lambda_", ctypes.c_float), ("beta", ctypes.c_float),
        ("dtype", ctypes.c_int32), ("head_criterion", ctypes.c_int32),
    ]


@dataclass
class Config:
    """Python view of kvec_config."""
    batch: int
    n_layers: int
    n_kv_heads: int
    n_q_heads: int
    head_dim: int
    seq_len: int
    window: int
    window_ext: int
    budget: int
    pool_kernel: int = 7
    n_adjust_heads: int = 3
    lam: float = 1.0
    beta: float = 0.25
    dtype: int = KVEC_BF16
    head_criterion: int = KVEC_HEADS_STD

    def c(self) -> kvec_config:
        return kvec_config(self.batch, self.n_layers, self.n_kv_heads, self.n_q_heads,
                           self.head_dim, self.seq_len, self.window, self.window_ext,
                           self.budget, self.pool_kernel, self.n_adjust_heads, self.lam,
                           self.beta, self.dtype, self.head_criterion)

    @classmethod
    def from_workload(cls, w, **over) -> "Config":
        kw = dict(batch=w.batch, n_layers=w.n_layers, n_kv_heads=w.n_kv_heads,
                  n_q_heads=w.n_q_heads, head_dim=w.head_dim, seq_len=w.seq_len,
                  window=w.window, window_ext=w.window_ext, budget=w.budget,
                  pool_kernel=w.pool_kernel, n_adjust_heads=w.n_adjust_heads, lam=w.lam,
                  beta=w.beta, dtype=KVEC_BF16 if w.dtype == "bf16" else KVEC_F32,
                  head_criterion=KVEC_HEADS_ENTROPY if getattr(w, "criterion", "std") == "entropy"
                  else KVEC_HEADS_STD)
        kw.update(over)
        return cls(**kw)

    @property
    def candidates(self) -> int:
        return self.seq_len - self.window

    @property
    def words(self) -> int:
        return (self.seq_len + 63) // 64


class kvec_attention_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_kv_heads", "n_q_heads", "head_dim", "q_len",
                                              "kv_len", "window", "n_sinks", "dtype")]


class kvec_paged_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_kv_heads", "n_q_heads", "head_dim",
                                              "page_size", "n_pages", "max_pages", "dtype")]


class kvec_paged_q8_config(ctypes.Structure):
    _fields_ = [("paged", kvec_paged_config), ("format", ctypes.c_int32)]


@dataclass(frozen=True)
class AttentionConfig:
    """Python view of kvec_attention_config."""
    batch: int
    n_kv_heads: int
    n_q_heads: int
    head_dim: int
    q_len: int
    kv_len: int
    window: int = 0
    n_sinks: int = 0
    dtype: int = KVEC_BF16

    def __post_init__(self):
        # what every call needs of the configuration, made once
        q, k = (self.batch, self.n_q_heads, self.q_len), (self.batch, self.n_kv_heads, self.kv_len)
        _fix(self, kvec_attention_config(self.batch, self.n_kv_heads, self.n_q_heads, self.head_dim,
                                         self.q_len, self.kv_len, self.window, self.n_sinks, self.dtype),
             q_shape=q + (self.head_dim,), k_shape=k + (self.head_dim,), lse_shape=q, len_shape=(self.batch,))

    def c(self) -> kvec_attention_config:
        return self._c

    def __reduce__(self):
        return _rebuild(self)


@dataclass(frozen=True)
class PagedConfig:
    """Python view of kvec_paged_config."""
    batch: int
    n_kv_heads: int
    n_q_heads: int
    head_dim: int
    page_size: int
    n_pages: int
    max_pages: int
    dtype: int = KVEC_BF16

    def __post_init__(self):
        meta = (self.n_pages, self.n_kv_heads, self.page_size)
        _fix(self, kvec_paged_config(self.batch, self.n_kv_heads, self.n_q_heads, self.head_dim,
                                     self.page_size, self.n_pages, self.max_pages, self.dtype),
             meta_shape=meta, pool_shape=meta + (self.head_dim,), table_shape=(self.batch, self.max_pages),
             len_shape=(self.batch,), lse_shape=(self.batch, self.n_q_heads),
             q_shape=(self.batch, self.n_q_heads, self.head_dim))

    def c(self) -> kvec_paged_config:
        return self._c

    def __reduce__(self):
        return _rebuild(self)


@dataclass(frozen=True)
class PagedQ8Config:
    """Python view of kvec_paged_q8_config: the fields of a PagedConfig, and the format."""
    batch: int
    n_kv_heads: int
    n_q_heads: int
    head_dim: int
    page_size: int
    n_pages: int
    max_pages: int
    dtype: int = KVEC_BF16
    format: int = KVEC_Q8_INT8

    def __post_init__(self):
        import torch
        p = PagedConfig(self.batch, self.n_kv_heads, self.n_q_heads, self.head_dim, self.page_size, self.n_pages,
                        self.max_pages, self.dtype)
        _fix(self, kvec_paged_q8_config(p.c(), self.format), **{n: getattr(p, n) for n in (
            "meta_shape", "pool_shape", "table_shape", "len_shape", "lse_shape", "q_shape")},
             code=torch.int8 if self.format == KVEC_Q8_INT8 else torch.float8_e4m3fn)

    def c(self) -> kvec_paged_q8_config:
        return self._c

    def __reduce__(self):
        return _rebuild(self)


def _rebuild(cfg):
    """Copies and pickles of a frozen configuration are made from its fields."""
    return type(cfg), tuple(getattr(cfg, f.name) for f in fields(cfg))


def _fix(cfg, c, **more) -> None:
    """Keeps the C view of a frozen configuration, a reference to it and its address, the types (of
    elements, float32, int32) and the shapes it implies."""
    import torch
    types = (torch.bfloat16 if cfg.dtype == KVEC_BF16 else torch.float32, torch.float32, torch.int32)
    for name, value in dict(_c=c, ref=ctypes.byref(c), addr=ctypes.addressof(c), types=types, **more).items():
        object.__setattr__(cfg, name, value)


_lib = None

EXPORTS = ["kvec_workspace_size", "kvec_score", "kvec_score_lse", "kvec_select_cover",
           "kvec_compact", "kvec_evict_layer", "kvec_evict_model", "kvec_evict_model_lse",
           "kvec_evict_layer_lse", "kvec_evict_model_scores", "kvec_evict_model_steps",
           "kvec_evict_model_lse_steps",
           "kvec_profile_points", "kvec_profile_points_lse", "kvec_coverage",
           "kvec_decode_workspace_size", "kvec_decode_attention", "kvec_decode_attention_noalloc",
           "kvec_prefill_workspace_size", "kvec_prefill_attention", "kvec_paged_append",
           "kvec_paged_decode_workspace_size", "kvec_paged_decode",
           "kvec_paged_evict_workspace_size", "kvec_paged_evict",
           "kvec_paged_decode_shared_workspace_size", "kvec_paged_decode_shared", "kvec_paged_append_q8",
           "kvec_paged_read_q8", "kvec_paged_decode_q8_workspace_size", "kvec_paged_decode_q8",
           "kvec_paged_evict_q8_workspace_size", "kvec_paged_evict_q8",
           "kvec_status_string"]


def load() -> ctypes.CDLL:
    """Load libkvec.so (building it first only if no build exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(kvec_config)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    I64x = ctypes.POINTER(ctypes.c_int64)
    lib.kvec_workspace_size.argtypes = [P, ctypes.POINTER(sz)]
    lib.kvec_score.argtypes = [P, vp, I64x, vp, I64x, vp, vp, vp, vp, sz, vp]
    lib.kvec_score_lse.argtypes = [P, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, vp, sz, vp]
    lib.kvec_select_cover.argtypes = [P, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.kvec_compact.argtypes = [P, vp, I64x, vp, I64x, vp, vp, vp, vp]
    lib.kvec_evict_layer.argtypes = [P, i32, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, vp, vp, sz, vp]
    lib.kvec_evict_model.argtypes = [P, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, vp, vp, sz, vp,
                                     ctypes.POINTER(vp)]
    lib.kvec_evict_layer_lse.argtypes = [P, i32, vp, I64x, vp, I64x, vp, I64x, vp, I64x, vp, vp,
                                         vp, vp, vp, sz, vp]
    lib.kvec_evict_model_lse.argtypes = [P, vp, I64x, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, vp,
                                         vp, sz, vp, ctypes.POINTER(vp)]
    lib.kvec_evict_model_scores.argtypes = [P, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, vp, vp,
                                            vp, vp, vp, vp, sz, vp]
    lib.kvec_evict_model_steps.argtypes = [P, i32, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, vp, vp,
                                           sz, vp]
    lib.kvec_evict_model_lse_steps.argtypes = [P, i32, vp, I64x, vp, I64x, vp, I64x, vp, I64x, vp, vp,
                                               vp, vp, vp, sz, vp]
    lib.kvec_decode_attention_noalloc.argtypes = [P, vp, I64x, vp, vp, I64x, i32, vp, vp, vp]
    lib.kvec_coverage.argtypes = [P, vp, i32, vp, vp]
    lib.kvec_decode_workspace_size.argtypes = [P, i32, ctypes.POINTER(sz)]
    lib.kvec_decode_attention.argtypes = [P, vp, I64x, vp, vp, I64x, i32, vp, vp, vp, sz, vp]
    lib.kvec_profile_points.argtypes = [P]
    lib.kvec_profile_points_lse.argtypes = [P]
    A, C = ctypes.POINTER(kvec_attention_config), ctypes.POINTER(kvec_paged_config)
    f32 = ctypes.c_float
    lib.kvec_prefill_workspace_size.argtypes = [A, ctypes.POINTER(sz)]
    lib.kvec_prefill_attention.argtypes = [A, vp, I64x, vp, I64x, vp, I64x, vp, vp, vp, I64x, vp, I64x,
                                           vp, sz, vp]
    lib.kvec_paged_append.argtypes = [C, i32, vp, I64x, vp, I64x, vp, I64x, vp, vp, f32, vp, vp, i32, vp,
                                      vp, I64x, vp, vp, I64x, vp, vp, vp]
    lib.kvec_paged_decode_workspace_size.argtypes = [C, i32, i32, ctypes.POINTER(sz)]
    lib.kvec_paged_decode.argtypes = [C, vp, I64x, vp, vp, I64x, vp, vp, i32, i32, i32, vp, vp, vp, vp,
                                      sz, vp]
    lib.kvec_paged_evict_workspace_size.argtypes = [C, i32, i32, ctypes.POINTER(sz)]
    lib.kvec_paged_evict.argtypes = [C, i32, i32, i32, vp, vp, I64x, vp, vp, vp, i32, vp, vp, vp, vp, vp,
                                     sz, vp]
    E = ctypes.POINTER(kvec_paged_q8_config)
    lib.kvec_paged_decode_shared_workspace_size.argtypes = [C, i32, i32, i32, ctypes.POINTER(sz)]
    lib.kvec_paged_decode_shared.argtypes = [C, vp, I64x, vp, vp, I64x, vp, i32, vp, i32, vp, vp, i32, i32, i32,
                                             vp, vp, vp, vp, sz, vp]
    lib.kvec_paged_append_q8.argtypes = [E, i32, vp, I64x, vp, I64x, vp, I64x, vp, vp, f32, vp, vp, i32, vp,
                                         vp, I64x, vp, vp, I64x, vp, vp, vp, vp, vp]
    lib.kvec_paged_read_q8.argtypes = [E, vp, vp, I64x, vp, vp, vp, vp, i32, vp, I64x, vp, I64x, vp]
    lib.kvec_paged_decode_q8_workspace_size.argtypes = [E, i32, i32, ctypes.POINTER(sz)]
    lib.kvec_paged_decode_q8.argtypes = [E, vp, I64x, vp, vp, I64x, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp,
                                         vp, sz, vp]
    lib.kvec_paged_evict_q8_workspace_size.argtypes = [E, i32, i32, ctypes.POINTER(sz)]
    lib.kvec_paged_evict_q8.argtypes = [E, i32, i32, i32, vp, vp, I64x, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp,
                                        vp, sz, vp]
    lib.kvec_status_string.argtypes = [ctypes.c_int]
    lib.kvec_status_string.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("kvec_status_string", "kvec_profile_points", "kvec_profile_points_lse"):
            getattr(lib, name).restype = ctypes.c_int
    lib.kvec_profile_points.restype = ctypes.c_int32
    lib.kvec_profile_points_lse.restype = ctypes.c_int32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().kvec_status_string(status).decode()


def _check(status: int, what: str) -> None:
    if status != KVEC_OK:
        raise KvecError(status, what)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _strides(t, n: int):
    """Element strides of the leading n dims of a tensor whose last dim is contiguous."""
    if t is None:
        return None
    assert t.stride(-1) == 1, "the head dimension must be contiguous"
    st = list(t.stride())[:n]
    return (ctypes.c_int64 * n)(*st)


def _lse_strides(t, n: int):
    """Element strides of the leading n dims of an fp32 lse tensor with contiguous rows."""
    import torch
    assert t.dtype == torch.float32, "lse must be float32"
    return _strides(t, n)


def _stream(stream) -> int:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def kvec_workspace_size(cfg: Config) -> int:
    out = ctypes.c_size_t(0)
    c = cfg.c()
    _check(load().kvec_workspace_size(ctypes.byref(c), ctypes.byref(out)), "kvec_workspace_size")
    return out.value


def kvec_score(cfg: Config, q_win, k, p_raw, p_ext_raw, imp, ws, stream=None) -> None:
    """q_win [b][HQ][O'][d], k [b][H][T][d]; outputs fp32 [b][H][Tc], [b][H][Tc], [b][Tc]."""
    c = cfg.c()
    _check(load().kvec_score(ctypes.byref(c), _ptr(q_win), _strides(q_win, 3), _ptr(k),
                             _strides(k, 3), _ptr(p_raw), _ptr(p_ext_raw), _ptr(imp), _ptr(ws),
                             ws.numel() * ws.element_size(), _stream(stream)), "kvec_score")


def kvec_score_lse(cfg: Config, q_win, lse, k, p_raw, p_ext_raw, imp, ws, stream=None) -> None:
    """As kvec_score, with the window rows' natural-log normalisers lse fp32 [b][HQ][O']."""
    c = cfg.c()
    _check(load().kvec_score_lse(ctypes.byref(c), _ptr(q_win), _strides(q_win, 3), _ptr(lse),
                                 _lse_strides(lse, 2), _ptr(k), _strides(k, 3), _ptr(p_raw),
                                 _ptr(p_ext_raw), _ptr(imp), _ptr(ws),
                                 ws.numel() * ws.element_size(), _stream(stream)), "kvec_score_lse")


def kvec_select_cover(cfg: Config, layer: int, p_raw, p_ext_raw, imp, cover_bits, idx,
                      htop_mask=None, ws=None, stream=None) -> None:
    c = cfg.c()
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(load().kvec_select_cover(ctypes.byref(c), layer, _ptr(p_raw), _ptr(p_ext_raw), _ptr(imp),
                                    _ptr(cover_bits), _ptr(idx), _ptr(htop_mask), _ptr(ws), nbytes,
                                    _stream(stream)), "kvec_select_cover")


def kvec_compact(cfg: Config, k, v, idx, k_out, v_out, stream=None) -> None:
    c = cfg.c()
    _check(load().kvec_compact(ctypes.byref(c), _ptr(k), _strides(k, 3), _ptr(v), _strides(v, 3),
                               _ptr(idx), _ptr(k_out), _ptr(v_out), _stream(stream)), "kvec_compact")


def kvec_evict_layer(cfg: Config, layer: int, q_win, k, v, cover_bits, idx, k_out, v_out, ws,
                     stream=None) -> None:
    c = cfg.c()
    _check(load().kvec_evict_layer(ctypes.byref(c), layer, _ptr(q_win), _strides(q_win, 3), _ptr(k),
                                   _strides(k, 3), _ptr(v), _strides(v, 3), _ptr(cover_bits),
                                   _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream(stream)),
           "kvec_evict_layer")


def kvec_evict_model(cfg: Config, q_win, k, v, cover_bits, idx, k_out, v_out, ws, stream=None,
                     events=None) -> None:
    """q_win [L][b][HQ][O'][d], k/v [L][b][H][T][d]; idx [L][b][H][B]; k_out/v_out [L][b][H][B][d].
    events: optional sequence of kvec_profile_points(cfg) raw hipEvent_t handles (ints)."""
    c = cfg.c()
    ev = None
    if events is not None:
        ev = (ctypes.c_void_p * len(events))(*events)
    _check(load().kvec_evict_model(ctypes.byref(c), _ptr(q_win), _strides(q_win, 4), _ptr(k),
                                   _strides(k, 4), _ptr(v), _strides(v, 4), _ptr(cover_bits),
                                   _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream(stream), ev),
           "kvec_evict_model")


def kvec_evict_model_steps(cfg: Config, q_win, k, v, cover_bits, idx, k_out, v_out, ws,
                           stream=None) -> None:
    """n independent steps in one pipelined call: q_win [n][L][b][HQ][O'][d], k/v
    [n][L][b][H][T][d] (any element strides, a step stride of 0 included);
    cover_bits [n][b][L][W], idx [n][L][b][H][B], k_out/v_out [n][L][b][H][B][d]
    contiguous."""
    c = cfg.c()
    n = k.shape[0]
    _check(load().kvec_evict_model_steps(ctypes.byref(c), n, _ptr(q_win), _strides(q_win, 5), _ptr(k),
                                         _strides(k, 5), _ptr(v), _strides(v, 5), _ptr(cover_bits),
                                         _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream(stream)),
           "kvec_evict_model_steps")


def kvec_evict_model_lse_steps(cfg: Config, q_win, lse, k, v, cover_bits, idx, k_out, v_out, ws,
                               stream=None) -> None:
    """As kvec_evict_model_steps, with the window rows' natural-log normalisers
    lse fp32 [n][L][b][HQ][O'] (any leading strides, rows contiguous)."""
    c = cfg.c()
    n = k.shape[0]
    _check(load().kvec_evict_model_lse_steps(ctypes.byref(c), n, _ptr(q_win), _strides(q_win, 5),
                                             _ptr(lse), _lse_strides(lse, 4), _ptr(k), _strides(k, 5),
                                             _ptr(v), _strides(v, 5), _ptr(cover_bits), _ptr(idx),
                                             _ptr(k_out), _ptr(v_out), _ptr(ws),
                                             ws.numel() * ws.element_size(), _stream(stream)),
           "kvec_evict_model_lse_steps")


def kvec_evict_model_scores(cfg: Config, q_win, k, v, cover_bits, idx, k_out, v_out, p_raw_out,
                            p_ext_out, imp_out, htop_out, ws, stream=None) -> None:
    """As kvec_evict_model, also writing each layer's scores before pooling:
    p_raw_out, p_ext_out fp32 [L][b][H][Tc] (P over O' for the H_top heads only),
    imp_out fp32 [L][b][Tc], htop_out int32/uint32 [L][b] (H_top bit masks)."""
    c = cfg.c()
    _check(load().kvec_evict_model_scores(ctypes.byref(c), _ptr(q_win), _strides(q_win, 4),
                                          _ptr(k), _strides(k, 4), _ptr(v), _strides(v, 4),
                                          _ptr(cover_bits), _ptr(idx), _ptr(k_out), _ptr(v_out),
                                          _ptr(p_raw_out), _ptr(p_ext_out), _ptr(imp_out),
                                          _ptr(htop_out), _ptr(ws),
                                          ws.numel() * ws.element_size(), _stream(stream)),
           "kvec_evict_model_scores")


def kvec_evict_layer_lse(cfg: Config, layer: int, q_win, lse, k, v, cover_bits, idx, k_out, v_out,
                         ws, stream=None) -> None:
    """As kvec_evict_layer, with the layer's natural-log row normalisers lse fp32 [b][HQ][O']."""
    c = cfg.c()
    _check(load().kvec_evict_layer_lse(ctypes.byref(c), layer, _ptr(q_win), _strides(q_win, 3),
                                       _ptr(lse), _lse_strides(lse, 2), _ptr(k), _strides(k, 3),
                                       _ptr(v), _strides(v, 3), _ptr(cover_bits), _ptr(idx),
                                       _ptr(k_out), _ptr(v_out), _ptr(ws),
                                       ws.numel() * ws.element_size(), _stream(stream)),
           "kvec_evict_layer_lse")


def kvec_evict_model_lse(cfg: Config, q_win, lse, k, v, cover_bits, idx, k_out, v_out, ws,
                         stream=None, events=None) -> None:
    """As kvec_evict_model, with the window rows' natural-log normalisers lse fp32
    [L][b][HQ][O'] (events: kvec_profile_points_lse(cfg) handles)."""
    c = cfg.c()
    ev = None
    if events is not None:
        ev = (ctypes.c_void_p * len(events))(*events)
    _check(load().kvec_evict_model_lse(ctypes.byref(c), _ptr(q_win), _strides(q_win, 4), _ptr(lse),
                                       _lse_strides(lse, 3), _ptr(k), _strides(k, 4), _ptr(v),
                                       _strides(v, 4), _ptr(cover_bits), _ptr(idx), _ptr(k_out),
                                       _ptr(v_out), _ptr(ws), ws.numel() * ws.element_size(),
                                       _stream(stream), ev),
           "kvec_evict_model_lse")


def kvec_profile_points_lse(cfg: Config) -> int:
    c = cfg.c()
    return int(load().kvec_profile_points_lse(ctypes.byref(c)))


def kvec_profile_points(cfg: Config) -> int:
    c = cfg.c()
    return int(load().kvec_profile_points(ctypes.byref(c)))


def kvec_coverage(cfg: Config, cover_bits, upto_layer: int, count, stream=None) -> None:
    c = cfg.c()
    _check(load().kvec_coverage(ctypes.byref(c), _ptr(cover_bits), upto_layer, _ptr(count),
                                _stream(stream)), "kvec_coverage")


def kvec_decode_workspace_size(cfg: Config, n_ctx: int) -> int:
    out = ctypes.c_size_t(0)
    c = cfg.c()
    _check(load().kvec_decode_workspace_size(ctypes.byref(c), n_ctx, ctypes.byref(out)),
           "kvec_decode_workspace_size")
    return out.value


def kvec_decode_attention(cfg: Config, q, k_cache, v_cache, out, ws, idx=None, n_ctx=None,
                          stream=None) -> None:
    """q [b][HQ][d]; k_cache/v_cache [b][H][n_ctx][d] (rows contiguous); out fp32 [b][HQ][d]."""
    c = cfg.c()
    n = k_cache.shape[2] if n_ctx is None else n_ctx
    assert k_cache.stride()[:2] == v_cache.stride()[:2], "K and V caches share their strides"
    assert k_cache.stride(2) == k_cache.shape[3] and v_cache.stride(2) == v_cache.shape[3], \
        "cache rows must be contiguous"
    _check(load().kvec_decode_attention(ctypes.byref(c), _ptr(q), _strides(q, 2), _ptr(k_cache),
                                        _ptr(v_cache), _strides(k_cache, 2), n, _ptr(idx),
                                        _ptr(out), _ptr(ws), ws.numel() * ws.element_size(),
                                        _stream(stream)), "kvec_decode_attention")


def kvec_decode_attention_noalloc(cfg: Config, q, k_cache, v_cache, out, idx=None, n_ctx=None,
                                  stream=None) -> None:
    """kvec_decode_attention without a workspace: the partial states use the
    library's fixed 4 MiB device scratch (calls overlapping on one device race)."""
    c = cfg.c()
    n = k_cache.shape[2] if n_ctx is None else n_ctx
    assert k_cache.stride()[:2] == v_cache.stride()[:2], "K and V caches share their strides"
    assert k_cache.stride(2) == k_cache.shape[3] and v_cache.stride(2) == v_cache.shape[3], \
        "cache rows must be contiguous"
    _check(load().kvec_decode_attention_noalloc(ctypes.byref(c), _ptr(q), _strides(q, 2),
                                                _ptr(k_cache), _ptr(v_cache), _strides(k_cache, 2),
                                                n, _ptr(idx), _ptr(out), _stream(stream)),
           "kvec_decode_attention_noalloc")


# The calls below are made once per layer and token, where a launch is shorter than the
# reading of a dozen tensors' attributes: the compiled module _kvec_bind checks and
# marshals them, and only where it finds something wrong Python goes through them again,
# for the message.

_bind = None


def _bound():
    """The compiled marshalling module, with the library's entry points."""
    global _bind
    if _bind is None:
        import torch  # noqa: F401  (its libraries, before the module that needs them)
        lib = load()
        if not os.path.exists(BIND_PATH):
            from . import build as _build
            _build.build_binding()
        from . import _kvec_bind
        at = lambda *names: (ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names)  # noqa: E731
        _kvec_bind.bind(*at("kvec_prefill_attention", "kvec_paged_append", "kvec_paged_decode", "kvec_paged_evict"))
        _kvec_bind.bind_forms(*at("kvec_paged_decode_shared", "kvec_paged_append_q8", "kvec_paged_read_q8",
                                  "kvec_paged_decode_q8", "kvec_paged_evict_q8"))
        _bind = _kvec_bind
    return _bind


def _serve(name: str, cfg, dev: int, stream, args, tensors) -> None:
    """_kvec_bind's call `name` with device `dev` current, on its current stream unless one
    is given.  tensors(): (what, tensor, shape, dtype, contiguous) of the arguments."""
    import torch
    status = -1
    if dev >= 0:
        fn = getattr(_bind or _bound(), name[5:])
        # the current stream's handle, without a Stream object around it
        st = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
        if dev == torch._C._cuda_getDevice():
            status = fn(cfg.addr, dev, st, *args)
        else:
            with torch.cuda.device(dev):
                status = fn(cfg.addr, dev, st, *args)
    if status > 0:
        raise KvecError(status, name)
    if status < 0:
        _refuse(name, tensors())


def _refuse(name: str, tensors) -> None:
    """Raises for the first tensor that is not what its entry says; what each is comes before
    where they are."""
    for what, t, shape, dtype, dense in tensors:
        assert t is not None, f"{name}: {what} must be given"
        assert tuple(t.shape) == tuple(shape), f"{name}: {what} must be {tuple(shape)}, not {tuple(t.shape)}"
        assert t.dtype == dtype, f"{name}: {what} must be {dtype}, not {t.dtype}"
        assert t.is_contiguous() if dense else t.stride(-1) == 1, \
            f"{name}: {what} must be contiguous" + ("" if dense else " in its last dimension")
    for what, t, *_ in tensors:
        assert t.is_cuda and t.device == tensors[0][1].device, f"{name}: {what} must be on the GPU of the other tensors"
    raise AssertionError(f"{name}: K and V pools must have the same strides, and a workspace be contiguous on their GPU")


def _other(name: str, kind):
    """Raises for a configuration of another kind: the compiled module reads it by address."""
    raise AssertionError(f"{name}: cfg must be a {kind.__name__}")


def _given(*entries) -> tuple:
    """Entries of the optional tensors that are there."""
    return tuple(e for e in entries if e[1] is not None)


def kvec_prefill_workspace_size(cfg: AttentionConfig) -> int:
    out = ctypes.c_size_t(0)
    _check(load().kvec_prefill_workspace_size(cfg.ref, ctypes.byref(out)), "kvec_prefill_workspace_size")
    return out.value


def kvec_prefill_attention(cfg: AttentionConfig, q, k, v, out, ws=None, lse=None, q_lens=None,
                           kv_lens=None, stream=None) -> None:
    """q, out [b][HQ][q_len][d]; k, v [b][H][kv_len][d] (any leading strides); lse fp32
    [b][HQ][q_len], rows contiguous; q_lens, kv_lens int32 [b].  ws may be None when
    kvec_prefill_workspace_size(cfg) is 0."""
    if not isinstance(cfg, AttentionConfig):
        _other("kvec_prefill_attention", AttentionConfig)
    dt, f32, i32 = cfg.types
    _serve("kvec_prefill_attention", cfg, q.get_device(), stream, (q, k, v, out, ws, lse, q_lens, kv_lens), lambda: (
        ("q", q, cfg.q_shape, dt, False), ("k", k, cfg.k_shape, dt, False), ("v", v, cfg.k_shape, dt, False),
        ("out", out, cfg.q_shape, dt, False), *_given(
            ("lse", lse, cfg.lse_shape, f32, False), ("q_lens", q_lens, cfg.len_shape, i32, True),
            ("kv_lens", kv_lens, cfg.len_shape, i32, True))))


def kvec_paged_append(cfg: PagedConfig, q, k, v, positions, slots, q_out, k_pool, v_pool, q_weight=None,
                      k_weight=None, eps=1e-6, inv_freq=None, acc=None, pos=None, stream=None) -> None:
    """q, q_out [n][HQ][d], k, v [n][H][d] (any token and head strides), positions int32
    [n], slots int64 [n] (page * page_size + row; -1: not stored), pools
    [n_pages][H][page_size][d]; weights [d] (None: no norm); inv_freq float64 [rot_dim / 2]
    (None: no rotation); acc fp32 and pos int32 [n_pages][H][page_size]."""
    if not isinstance(cfg, PagedConfig):
        _other("kvec_paged_append", PagedConfig)
    def tensors():
        import torch
        (dt, f32, i32), n, d = cfg.types, 0 if q is None else q.shape[0], cfg.head_dim
        half = 0 if inv_freq is None else inv_freq.shape[0]
        return (("k_pool", k_pool, cfg.pool_shape, dt, False), ("v_pool", v_pool, cfg.pool_shape, dt, False),
                ("q", q, (n, cfg.n_q_heads, d), dt, False), ("k", k, (n, cfg.n_kv_heads, d), dt, False),
                ("v", v, (n, cfg.n_kv_heads, d), dt, False), ("q_out", q_out, (n, cfg.n_q_heads, d), dt, False),
                ("positions", positions, (n,), i32, True), ("slots", slots, (n,), torch.int64, True), *_given(
                    ("q_weight", q_weight, (d,), dt, True), ("k_weight", k_weight, (d,), dt, True),
                    ("inv_freq", inv_freq, (half,), torch.float64, True), ("acc", acc, cfg.meta_shape, f32, True),
                    ("pos", pos, cfg.meta_shape, i32, True)))
    _serve("kvec_paged_append", cfg, k_pool.get_device(), stream, (
        q, k, v, positions, slots, q_out, k_pool, v_pool, q_weight, k_weight, eps, inv_freq, acc, pos), tensors)


def _max_len(cfg: PagedConfig, max_len) -> int:
    return cfg.max_pages * cfg.page_size if max_len is None else max_len


def kvec_paged_decode_workspace_size(cfg: PagedConfig, max_len: int | None = None,
                                     with_acc: bool = False) -> int:
    out = ctypes.c_size_t(0)
    _check(load().kvec_paged_decode_workspace_size(cfg.ref, _max_len(cfg, max_len), int(with_acc),
                                                   ctypes.byref(out)), "kvec_paged_decode_workspace_size")
    return out.value


def kvec_paged_decode(cfg: PagedConfig, q, k_pool, v_pool, page_table, lens, out, ws, max_len=None,
                      window=0, n_sinks=0, lse=None, acc=None, stream=None) -> None:
    """q [b][HQ][d]; pools [n_pages][H][page_size][d] (K and V with the same strides);
    page_table int32 [b][max_pages]; lens int32 [b]; out fp32 [b][HQ][d]; lse fp32
    [b][HQ]; acc fp32 [n_pages][H][page_size].  max_len None: every slot of the table."""
    if not isinstance(cfg, PagedConfig):
        _other("kvec_paged_decode", PagedConfig)
    dt, f32, i32 = cfg.types
    n = cfg.max_pages * cfg.page_size if max_len is None else max_len
    _serve("kvec_paged_decode", cfg, q.get_device(), stream, (
        q, k_pool, v_pool, page_table, lens, out, ws, n, window, n_sinks, lse, acc), lambda: (
        ("q", q, cfg.q_shape, dt, False), ("k_pool", k_pool, cfg.pool_shape, dt, False),
        ("v_pool", v_pool, cfg.pool_shape, dt, False), ("page_table", page_table, cfg.table_shape, i32, True),
        ("lens", lens, cfg.len_shape, i32, True), ("out", out, cfg.q_shape, f32, True), *_given(
            ("lse", lse, cfg.lse_shape, f32, True), ("acc", acc, cfg.meta_shape, f32, True))))


def kvec_paged_evict_workspace_size(cfg: PagedConfig, max_len: int | None, budget: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().kvec_paged_evict_workspace_size(cfg.ref, _max_len(cfg, max_len), budget, ctypes.byref(out)),
           "kvec_paged_evict_workspace_size")
    return out.value


def kvec_paged_evict(cfg: PagedConfig, budget: int, k_pool, v_pool, page_table, lens, n_seen, acc, pos,
                     lens_out, ws, window=0, n_sinks=0, kept=None, max_len=None, stream=None) -> None:
    """Pools and tables as in kvec_paged_decode; acc fp32 and pos int32
    [n_pages][H][page_size]; lens, n_seen, lens_out int32 [b] (lens_out may be lens);
    kept int32 [b][H][budget]."""
    if not isinstance(cfg, PagedConfig):
        _other("kvec_paged_evict", PagedConfig)
    dt, f32, i32 = cfg.types
    n = cfg.max_pages * cfg.page_size if max_len is None else max_len
    _serve("kvec_paged_evict", cfg, k_pool.get_device(), stream, (
        budget, k_pool, v_pool, page_table, lens, n_seen, acc, pos, lens_out, ws, window, n_sinks, kept, n), lambda: (
        ("k_pool", k_pool, cfg.pool_shape, dt, False), ("v_pool", v_pool, cfg.pool_shape, dt, False),
        ("page_table", page_table, cfg.table_shape, i32, True), ("lens", lens, cfg.len_shape, i32, True),
        ("n_seen", n_seen, cfg.len_shape, i32, True), ("lens_out", lens_out, cfg.len_shape, i32, True),
        ("acc", acc, cfg.meta_shape, f32, True), ("pos", pos, cfg.meta_shape, i32, True),
        *_given(("kept", kept, (cfg.batch, cfg.n_kv_heads, budget), i32, True))))


def kvec_paged_decode_shared_workspace_size(cfg: PagedConfig, max_prefix: int, max_len: int | None = None,
                                            with_acc: bool = False) -> int:
    out = ctypes.c_size_t(0)
    _check(load().kvec_paged_decode_shared_workspace_size(cfg.ref, max_prefix, _max_len(cfg, max_len), int(with_acc),
                                                          ctypes.byref(out)),
           "kvec_paged_decode_shared_workspace_size")
    return out.value


def kvec_paged_decode_shared(cfg: PagedConfig, q, k_pool, v_pool, prefix_pages, prefix_len, page_table, lens, out,
                             ws, max_prefix=None, max_len=None, window=0, n_sinks=0, lse=None, acc=None,
                             stream=None) -> None:
    """As kvec_paged_decode, every sequence behind the prefix_len (int32 [1]) slots of the
    pages prefix_pages (int32 [n]); lens and max_len count the slots behind it (a negative
    length: no sequence).  max_prefix None: every slot of the prefix's pages."""
    if not isinstance(cfg, PagedConfig):
        _other("kvec_paged_decode_shared", PagedConfig)
    dt, f32, i32 = cfg.types
    n = cfg.max_pages * cfg.page_size if max_len is None else max_len
    pages = prefix_pages.shape[0] if prefix_pages is not None and prefix_pages.dim() else 0
    p = pages * cfg.page_size if max_prefix is None else max_prefix
    _serve("kvec_paged_decode_shared", cfg, q.get_device(), stream, (
        q, k_pool, v_pool, prefix_pages, prefix_len, page_table, lens, out, ws, p, n, window, n_sinks, lse, acc), lambda: (
        ("q", q, cfg.q_shape, dt, False), ("k_pool", k_pool, cfg.pool_shape, dt, False),
        ("v_pool", v_pool, cfg.pool_shape, dt, False), ("prefix_pages", prefix_pages, (pages,), i32, True),
        ("prefix_len", prefix_len, (1,), i32, True), ("page_table", page_table, cfg.table_shape, i32, True),
        ("lens", lens, cfg.len_shape, i32, True), ("out", out, cfg.q_shape, f32, True), *_given(
            ("lse", lse, cfg.lse_shape, f32, True), ("acc", acc, cfg.meta_shape, f32, True))))


def _q8_pools(cfg: PagedQ8Config, k_pool, v_pool, k_scale, v_scale) -> tuple:
    """Entries of an 8-bit cache's tensors."""
    return (("k_pool", k_pool, cfg.pool_shape, cfg.code, False), ("v_pool", v_pool, cfg.pool_shape, cfg.code, False),
            ("k_scale", k_scale, cfg.meta_shape, cfg.types[1], True), ("v_scale", v_scale, cfg.meta_shape, cfg.types[1], True))


def kvec_paged_append_q8(cfg: PagedQ8Config, q, k, v, positions, slots, q_out, k_pool, v_pool, k_scale, v_scale,
                         q_weight=None, k_weight=None, eps=1e-6, inv_freq=None, acc=None, pos=None,
                         stream=None) -> None:
    """As kvec_paged_append, into pools int8 or float8_e4m3fn (cfg.format)
    [n_pages][H][page_size][d] with scales fp32 [n_pages][H][page_size]."""
    if not isinstance(cfg, PagedQ8Config):
        _other("kvec_paged_append_q8", PagedQ8Config)
    def tensors():
        import torch
        (dt, f32, i32), n, d = cfg.types, 0 if q is None else q.shape[0], cfg.head_dim
        half = 0 if inv_freq is None else inv_freq.shape[0]
        return (*_q8_pools(cfg, k_pool, v_pool, k_scale, v_scale),
                ("q", q, (n, cfg.n_q_heads, d), dt, False), ("k", k, (n, cfg.n_kv_heads, d), dt, False),
                ("v", v, (n, cfg.n_kv_heads, d), dt, False), ("q_out", q_out, (n, cfg.n_q_heads, d), dt, False),
                ("positions", positions, (n,), i32, True), ("slots", slots, (n,), torch.int64, True), *_given(
                    ("q_weight", q_weight, (d,), dt, True), ("k_weight", k_weight, (d,), dt, True),
                    ("inv_freq", inv_freq, (half,), torch.float64, True), ("acc", acc, cfg.meta_shape, f32, True),
                    ("pos", pos, cfg.meta_shape, i32, True)))
    _serve("kvec_paged_append_q8", cfg, k_pool.get_device(), stream, (
        q, k, v, positions, slots, q_out, k_pool, v_pool, k_scale, v_scale, q_weight, k_weight, eps, inv_freq, acc,
        pos), tensors)


def kvec_paged_read_q8(cfg: PagedQ8Config, k_pool, v_pool, k_scale, v_scale, page_table, lens, k_out, v_out,
                       stream=None) -> None:
    """The rows of slots 0..lens[b] of every sequence: k_out, v_out [b][H][max_len][d] of
    cfg.dtype (any leading strides), max_len their own."""
    if not isinstance(cfg, PagedQ8Config):
        _other("kvec_paged_read_q8", PagedQ8Config)
    def tensors():
        dt, _, i32 = cfg.types
        n = k_out.shape[2] if k_out is not None and k_out.dim() > 2 else 0
        shape = (cfg.batch, cfg.n_kv_heads, n, cfg.head_dim)
        return (*_q8_pools(cfg, k_pool, v_pool, k_scale, v_scale), ("page_table", page_table, cfg.table_shape, i32, True),
                ("lens", lens, cfg.len_shape, i32, True), ("k_out", k_out, shape, dt, False), ("v_out", v_out, shape, dt, False))
    _serve("kvec_paged_read_q8", cfg, k_pool.get_device(), stream, (
        k_pool, v_pool, k_scale, v_scale, page_table, lens, k_out, v_out), tensors)


def kvec_paged_decode_q8_workspace_size(cfg: PagedQ8Config, max_len: int | None = None,
                                        with_acc: bool = False) -> int:
    out = ctypes.c_size_t(0)
    _check(load().kvec_paged_decode_q8_workspace_size(cfg.ref, _max_len(cfg, max_len), int(with_acc),
                                                      ctypes.byref(out)), "kvec_paged_decode_q8_workspace_size")
    return out.value


def kvec_paged_decode_q8(cfg: PagedQ8Config, q, k_pool, v_pool, k_scale, v_scale, page_table, lens, out, ws,
                         max_len=None, window=0, n_sinks=0, lse=None, acc=None, stream=None) -> None:
    """As kvec_paged_decode, over pools and scales as in kvec_paged_append_q8."""
    if not isinstance(cfg, PagedQ8Config):
        _other("kvec_paged_decode_q8", PagedQ8Config)
    dt, f32, i32 = cfg.types
    n = cfg.max_pages * cfg.page_size if max_len is None else max_len
    _serve("kvec_paged_decode_q8", cfg, q.get_device(), stream, (
        q, k_pool, v_pool, k_scale, v_scale, page_table, lens, out, ws, n, window, n_sinks, lse, acc), lambda: (
        ("q", q, cfg.q_shape, dt, False), *_q8_pools(cfg, k_pool, v_pool, k_scale, v_scale),
        ("page_table", page_table, cfg.table_shape, i32, True), ("lens", lens, cfg.len_shape, i32, True),
        ("out", out, cfg.q_shape, f32, True), *_given(
            ("lse", lse, cfg.lse_shape, f32, True), ("acc", acc, cfg.meta_shape, f32, True))))


def kvec_paged_evict_q8_workspace_size(cfg: PagedQ8Config, max_len: int | None, budget: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().kvec_paged_evict_q8_workspace_size(cfg.ref, _max_len(cfg, max_len), budget, ctypes.byref(out)),
           "kvec_paged_evict_q8_workspace_size")
    return out.value


def kvec_paged_evict_q8(cfg: PagedQ8Config, budget: int, k_pool, v_pool, k_scale, v_scale, page_table, lens, n_seen,
                        acc, pos, lens_out, ws, window=0, n_sinks=0, kept=None, max_len=None, stream=None) -> None:
    """As kvec_paged_evict, over pools and scales as in kvec_paged_append_q8."""
    if not isinstance(cfg, PagedQ8Config):
        _other("kvec_paged_evict_q8", PagedQ8Config)
    _, f32, i32 = cfg.types
    n = cfg.max_pages * cfg.page_size if max_len is None else max_len
    _serve("kvec_paged_evict_q8", cfg, k_pool.get_device(), stream, (
        budget, k_pool, v_pool, k_scale, v_scale, page_table, lens, n_seen, acc, pos, lens_out, ws, window, n_sinks, kept, n),
        lambda: (
        *_q8_pools(cfg, k_pool, v_pool, k_scale, v_scale),
        ("page_table", page_table, cfg.table_shape, i32, True), ("lens", lens, cfg.len_shape, i32, True),
        ("n_seen", n_seen, cfg.len_shape, i32, True), ("lens_out", lens_out, cfg.len_shape, i32, True),
        ("acc", acc, cfg.meta_shape, f32, True), ("pos", pos, cfg.meta_shape, i32, True),
        *_given(("kept", kept, (cfg.batch, cfg.n_kv_heads, budget), i32, True))))
