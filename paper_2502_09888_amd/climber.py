"""ctypes binding of include/climber.h.  Function names equal the C entry points; tensors are
passed as raw device pointers (``tensor.data_ptr()``), streams as ``torch.cuda.Stream`` or None
(= torch's current stream).  No arithmetic happens here."""
from __future__ import annotations

import ctypes as C
import os
from importlib.machinery import EXTENSION_SUFFIXES
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libclimber.so")
_NATIVE_PATH = os.path.join(_HERE, "_native" + EXTENSION_SUFFIXES[0])  # (another interpreter's has another name)

F32, BF16 = 0, 1
MODE_HISTORY, MODE_CANDIDATE = 0, 1
HIST_CAUSAL, HIST_TWO_KERNEL, QKV_VIA_ROWS = 1, 2, 4


class ClimberError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: error {code}: {climber_strerror(code)}")


class Config(C.Structure):
    """Mirror of ``climber_config``."""
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "d_head", "d_ffn",
                                         "n_scen", "n_beh", "sub_len", "dtype", "flags")] + \
               [("qk_scale", C.c_float), ("rms_eps", C.c_float)]

    def __init__(self, n_layers=1, d_model=0, n_heads=1, d_head=64, d_ffn=0, n_scen=1, n_beh=1,
                 sub_len=0, dtype=BF16, flags=0, qk_scale=1.0, rms_eps=1e-6):
        super().__init__(n_layers, d_model or n_heads * d_head, n_heads, d_head, d_ffn, n_scen,
                         n_beh, sub_len, dtype, flags, qk_scale, rms_eps)


class LayerWeights(C.Structure):
    """Mirror of ``climber_layer_weights`` (device pointers)."""
    _fields_ = [(n, C.c_void_p) for n in ("g1", "wqkv", "wo", "g2", "w1", "w2")]


class RelBias(C.Structure):
    """Mirror of ``climber_rel_bias`` (device pointers).  Build with ``rel_bias(...)``."""
    _fields_ = [("pos_table", C.c_void_p), ("time_table", C.c_void_p), ("n_pos", C.c_int32),
                ("n_time", C.c_int32), ("hist_pos", C.c_void_p), ("hist_ts", C.c_void_p),
                ("cand_pos", C.c_void_p), ("cand_ts", C.c_void_p)]


class BgfWeights(C.Structure):
    """Mirror of ``climber_bgf_weights``."""
    _fields_ = [("atl", LayerWeights), ("w_down", C.c_void_p), ("w_up", C.c_void_p), ("w_head", C.c_void_p),
                ("tau_scen", C.c_void_p), ("b_head", C.c_float), ("n_blocks", C.c_int32), ("d_gate", C.c_int32)]


class PagedKV(C.Structure):
    """Mirror of ``climber_paged_kv`` (device pointers).  Build with ``paged_kv(...)``."""
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "mass", "stamp", "page_table", "len")] + \
               [(n, C.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "n_seqs", "table_ld", "max_len", "d_head", "elem_bytes")]
    _device = None  # the CUDA device of its tensors (-1: they are in host memory that is not pinned), if it was made from tensors


class PagedKV8(C.Structure):
    """Mirror of ``climber_paged_kv8`` (device pointers).  Build with ``paged_kv8(...)``; its ``kv`` goes to ``climber_check_paged``."""
    _fields_ = [("kv", PagedKV), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]
    _device = None  # as PagedKV's


class PagePool(C.Structure):
    """Mirror of ``climber_page_pool`` (device pointers).  Build with ``page_pool(...)``."""
    _fields_ = [(n, C.c_void_p) for n in ("refs", "page_table", "held", "len")] + [(n, C.c_int32) for n in ("n_pages", "page_size", "n_seqs", "table_ld")]
    _device = None  # as PagedKV's


class RotaryPlan(C.Structure):
    """Mirror of ``climber_rotary_plan`` (device pointer).  Build with ``rotary(...)``."""
    _fields_ = [("freq", C.c_void_p)] + [(n, C.c_int32) for n in ("rot_dims", "interleaved", "inverse")] + [("scale", C.c_float)]
    _device = None  # as PagedKV's


class _Weights(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("layers", C.POINTER(LayerWeights)), ("packed", C.c_void_p)]


_lib = None
_native = None   # csrc/binding.c: the attention calls without ctypes' conversions


def library_path() -> str:
    return _LIB_PATH


def _built(path: str) -> None:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2502_09888_amd.build`"
                          " (there is no CPU fallback)")


def load_library():
    """Load libclimber.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    _built(_LIB_PATH)
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    cfgp = C.POINTER(Config)
    lib.climber_strerror.restype = C.c_char_p
    lib.climber_strerror.argtypes = [C.c_int]
    lib.climber_kv_cache_bytes.restype = sz
    lib.climber_kv_cache_bytes.argtypes = [cfgp, i32, C.POINTER(i32)]
    lib.climber_kv_cache_create.restype = C.c_int
    lib.climber_kv_cache_create.argtypes = [cfgp, i32, C.POINTER(i32), C.POINTER(i32), vp, sz,
                                            C.POINTER(vp)]
    lib.climber_kv_cache_destroy.restype = C.c_int
    lib.climber_kv_cache_destroy.argtypes = [vp]
    lib.climber_kv_cache_rows.restype = i64
    lib.climber_kv_cache_rows.argtypes = [vp]
    lib.climber_attn_history.restype = C.c_int
    lib.climber_attn_history.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.climber_attn_sumi.restype = C.c_int
    lib.climber_attn_sumi.argtypes = [cfgp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.climber_attn_history_bias.restype = C.c_int
    lib.climber_attn_history_bias.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i32, vp, C.POINTER(RelBias), vp]
    lib.climber_attn_sumi_bias.restype = C.c_int
    lib.climber_attn_sumi_bias.argtypes = [cfgp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp,
                                           C.POINTER(RelBias), vp]
    lib.climber_check_inputs.restype = C.c_int
    lib.climber_check_inputs.argtypes = [cfgp, vp, vp, vp, vp, i32, vp, i32, i32, vp, vp]
    lib.climber_workspace_bytes.restype = sz
    lib.climber_workspace_bytes.argtypes = [cfgp, i64]
    lib.climber_packed_weights_bytes.restype = sz
    lib.climber_packed_weights_bytes.argtypes = [cfgp]
    lib.climber_pack_weights.restype = C.c_int
    lib.climber_pack_weights.argtypes = [cfgp, C.POINTER(_Weights), vp, sz, vp]
    lib.climber_layer_forward.restype = C.c_int
    lib.climber_layer_forward.argtypes = [cfgp, C.POINTER(LayerWeights), vp, i32, i32, vp, vp, vp,
                                          vp, vp, vp, i32, i32, vp, sz, vp]
    lib.climber_history_encode.restype = C.c_int
    lib.climber_history_encode.argtypes = [cfgp, C.POINTER(_Weights), vp, vp, vp, vp, vp, vp, sz,
                                           vp]
    lib.climber_sumi_score.restype = C.c_int
    lib.climber_sumi_score.argtypes = [cfgp, C.POINTER(_Weights), vp, vp, vp, vp, i32, i32, vp,
                                       vp, vp, vp, sz, vp]
    lib.climber_bgf_workspace_bytes.restype = sz
    lib.climber_bgf_workspace_bytes.argtypes = [cfgp, i32, i32, i64]
    lib.climber_bgf_score.restype = C.c_int
    lib.climber_bgf_score.argtypes = [cfgp, C.POINTER(BgfWeights), vp, vp, i32, vp, vp, vp, sz, vp]
    lib.climber_sumi_forward.restype = C.c_int
    lib.climber_sumi_forward.argtypes = [cfgp, C.POINTER(_Weights), vp, vp, vp, vp, vp, vp, i32, i32, vp, vp,
                                         vp, vp, vp, vp, sz, vp]
    lib.climber_sumi_score_static.restype = C.c_int
    lib.climber_sumi_score_static.argtypes = [cfgp, C.POINTER(_Weights), vp, vp, vp, vp, i32, i32, vp,
                                              vp, vp, vp]
    pkv = C.POINTER(PagedKV)
    lib.climber_paged_workspace_bytes.restype = sz
    lib.climber_paged_workspace_bytes.argtypes = [cfgp, pkv, i32, i32]
    lib.climber_attn_history_paged.restype = C.c_int
    lib.climber_attn_history_paged.argtypes = [cfgp, vp, pkv, vp, i64, vp, vp, i64, vp, i32, i32, vp, vp, vp, vp, i64, vp, sz, vp]
    lib.climber_attn_sumi_paged.restype = C.c_int
    lib.climber_attn_sumi_paged.argtypes = [cfgp, vp, pkv, vp, i64, vp, vp, i64, vp, i32, i32, vp, vp, vp, i64, vp, sz, vp]
    lib.climber_paged_evict.restype = C.c_int
    lib.climber_paged_evict.argtypes = [cfgp, pkv, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.climber_check_paged.restype = C.c_int
    lib.climber_check_paged.argtypes = [cfgp, pkv, vp, i32, i32, i32, vp, vp]
    pkv8 = C.POINTER(PagedKV8)
    lib.climber_paged8_workspace_bytes.restype = sz
    lib.climber_paged8_workspace_bytes.argtypes = [cfgp, pkv8, i32, i32]
    lib.climber_attn_history_paged8.restype = C.c_int
    lib.climber_attn_history_paged8.argtypes = [cfgp, vp, pkv8, vp, i64, vp, vp, i64, vp, i32, i32, vp, vp, vp, vp, i64, vp, sz, vp]
    lib.climber_attn_sumi_paged8.restype = C.c_int
    lib.climber_attn_sumi_paged8.argtypes = [cfgp, vp, pkv8, vp, i64, vp, vp, i64, vp, i32, i32, vp, vp, vp, i64, vp, sz, vp]
    pool = C.POINTER(PagePool)
    lib.climber_pages_workspace_bytes.restype = sz
    lib.climber_pages_workspace_bytes.argtypes = [pool]
    for name, types in (("climber_pages_fork", [pool, vp, vp, vp, vp, sz, vp]), ("climber_pages_extend", [pool, vp, vp, vp, vp, vp, sz, vp]),
                        ("climber_pages_compact", [pool, vp, vp, vp, vp, sz, vp]), ("climber_paged_copy", [cfgp, pkv, vp, vp, i32, vp]),
                        ("climber_paged8_copy", [cfgp, pkv8, vp, vp, i32, vp])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = C.c_int, types
    f64 = C.c_double
    lib.climber_rotary_frequencies.restype = C.c_int
    lib.climber_rotary_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, C.POINTER(f64), C.POINTER(C.c_float)]
    lib.climber_rotary.restype = C.c_int
    lib.climber_rotary.argtypes = [cfgp, C.POINTER(RotaryPlan), vp, i64, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    try:
        _load_native(lib)
    except ImportError:  # the host's calls do without; an attention call raises it
        pass
    _lib = lib
    return lib


def _load_native(lib):
    """csrc/binding.c over the library's attention calls."""
    global _native
    _built(_NATIVE_PATH)
    from . import _native as native
    try:
        import torch
        current = torch.cuda.current_device, torch._C._cuda_getCurrentRawStream
    except (ImportError, AttributeError):  # then a call names its stream, or _stream raises it
        current = None, None
    native.bind(*(C.cast(f, C.c_void_p).value for f in (lib.climber_attn_history, lib.climber_attn_sumi, lib.climber_attn_history_bias,
                                                        lib.climber_attn_sumi_bias)),
                Config, RelBias, *current,
                *(C.cast(f, C.c_void_p).value for f in (lib.climber_attn_history_paged, lib.climber_attn_sumi_paged, lib.climber_paged_evict)),
                PagedKV, *(C.cast(f, C.c_void_p).value for f in (lib.climber_attn_history_paged8, lib.climber_attn_sumi_paged8)), PagedKV8)
    if current[0] is not None:
        native.bind_pages(*(C.cast(f, C.c_void_p).value for f in (lib.climber_pages_fork, lib.climber_pages_extend, lib.climber_pages_compact,
                                                                  lib.climber_paged_copy, lib.climber_paged8_copy, lib.climber_rotary)),
                          PagePool, RotaryPlan, torch.bfloat16, torch.float32, torch.int32)
    _native = native
    return native


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        # The handle by itself: torch.cuda.current_stream() builds a Stream object around it, 2.9 of a small call's 7.9 us
        # on the host (0.3 this way; two fp32 calls of one small user 15.6 us as a pass, 10.9 this way).
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _i32arr(xs: Sequence[int]):
    return (C.c_int32 * len(xs))(*[int(x) for x in xs])


def _ok(code: int, where: str):
    if code != 0:
        raise ClimberError(code, where)


def climber_strerror(code: int) -> str:
    return load_library().climber_strerror(int(code)).decode()


def climber_kv_cache_bytes(cfg: Config, hist_len_padded: Sequence[int]) -> int:
    return int(load_library().climber_kv_cache_bytes(C.byref(cfg), len(hist_len_padded),
                                                     _i32arr(hist_len_padded)))


class KVCache:
    """Owner of a ``climber_kv_cache`` handle (the device buffer stays with the caller)."""

    def __init__(self, handle: int, dev_buf):
        self.handle = handle
        self.dev_buf = dev_buf  # keeps the tensor alive

    def __del__(self):
        try:
            climber_kv_cache_destroy(self)
        except Exception:
            pass


def climber_kv_cache_create(cfg: Config, hist_len: Sequence[int], hist_len_padded: Sequence[int],
                            dev_buf, nbytes: Optional[int] = None) -> KVCache:
    B = len(hist_len)
    if len(hist_len_padded) != B:
        raise ValueError("hist_len and hist_len_padded differ in length")
    if nbytes is None:
        nbytes = dev_buf.numel() * dev_buf.element_size()
    out = C.c_void_p()
    _ok(load_library().climber_kv_cache_create(C.byref(cfg), B, _i32arr(hist_len),
                                               _i32arr(hist_len_padded), _ptr(dev_buf), nbytes,
                                               C.byref(out)), "climber_kv_cache_create")
    return KVCache(out.value, dev_buf)


def climber_kv_cache_destroy(cache: KVCache) -> None:
    if cache.handle:
        load_library().climber_kv_cache_destroy(cache.handle)
        cache.handle = None


def climber_kv_cache_rows(cache: KVCache) -> int:
    return int(load_library().climber_kv_cache_rows(cache.handle))


def climber_attn_history(cfg: Config, tau_layer, q, k, v, scen, beh, cache: KVCache, layer: int,
                         o_hist=None, stream=None) -> None:
    code = (_native or _load_native(load_library())).attn_history(cfg, tau_layer, q, k, v, scen, beh, cache.handle, layer, o_hist, stream)
    if code is None:
        code = load_library().climber_attn_history(C.byref(cfg), _ptr(tau_layer), _ptr(q), _ptr(k), _ptr(v), _ptr(scen), _ptr(beh),
                                                   cache.handle, layer, _ptr(o_hist), _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_history")


def climber_attn_sumi(cfg: Config, tau_layer, cache: KVCache, layer: int, q_c, k_c, v_c, cand_off,
                      m_total: int, m_max: int, cand_scen, cand_beh, o_c, stream=None) -> None:
    code = (_native or _load_native(load_library())).attn_sumi(cfg, tau_layer, cache.handle, layer, q_c, k_c, v_c, cand_off, m_total, m_max,
                                                               cand_scen, cand_beh, o_c, stream)
    if code is None:
        code = load_library().climber_attn_sumi(C.byref(cfg), _ptr(tau_layer), cache.handle, layer, _ptr(q_c), _ptr(k_c), _ptr(v_c),
                                                _ptr(cand_off), m_total, m_max, _ptr(cand_scen), _ptr(cand_beh), _ptr(o_c), _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_sumi")


BAD_SCEN, BAD_BEH, BAD_TAU, BAD_OFFSETS, BAD_M_MAX, BAD_PAGE, BAD_LEN = 1, 2, 4, 8, 16, 32, 64
POOL_FULL, BAD_SEQ = 128, 256


def climber_check_inputs(cfg: Config, tau_layer, scen, beh, cache: Optional[KVCache], m_total: int,
                         cand_off, B_cand: int, m_max: int, status, stream=None) -> None:
    """Device-side check of ids / offsets / temperatures; ORs BAD_* bits into status (int32 tensor)."""
    _ok(load_library().climber_check_inputs(C.byref(cfg), _ptr(tau_layer), _ptr(scen), _ptr(beh),
                                            cache.handle if cache is not None else None, m_total,
                                            _ptr(cand_off), B_cand, m_max, _ptr(status),
                                            _stream(stream)), "climber_check_inputs")


def climber_workspace_bytes(cfg: Config, max_rows: int) -> int:
    return int(load_library().climber_workspace_bytes(C.byref(cfg), max_rows))


def _layer_struct(lw) -> LayerWeights:
    if isinstance(lw, LayerWeights):
        return lw
    return LayerWeights(*[_ptr(lw[n]) for n in ("g1", "wqkv", "wo", "g2", "w1", "w2")])


def _weights_struct(layers, packed=None):
    arr = (LayerWeights * len(layers))(*[_layer_struct(l) for l in layers])
    return _Weights(len(layers), arr, _ptr(packed)), arr


def climber_packed_weights_bytes(cfg: Config) -> int:
    return int(load_library().climber_packed_weights_bytes(C.byref(cfg)))


def climber_pack_weights(cfg: Config, layers, packed, stream=None) -> None:
    """Bring the weights into the form the projections read, once; pass the buffer as `packed` to
    climber_history_encode / climber_sumi_score."""
    w, keep = _weights_struct(layers)
    _ok(load_library().climber_pack_weights(C.byref(cfg), C.byref(w), _ptr(packed),
                                            packed.numel() * packed.element_size(), _stream(stream)),
        "climber_pack_weights")


def climber_layer_forward(cfg: Config, layer_weights, tau_layer, layer: int, mode: int,
                          cache: KVCache, x_in, x_out, scen, beh, cand_off, m_total: int,
                          m_max: int, workspace, stream=None) -> None:
    lw = _layer_struct(layer_weights)
    _ok(load_library().climber_layer_forward(
        C.byref(cfg), C.byref(lw), _ptr(tau_layer), layer, mode, cache.handle, _ptr(x_in),
        _ptr(x_out), _ptr(scen), _ptr(beh), _ptr(cand_off), m_total, m_max, _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)), "climber_layer_forward")


def climber_history_encode(cfg: Config, layers, tau, x_hist, scen, beh, cache: KVCache, workspace,
                           stream=None, packed=None) -> None:
    w, keep = _weights_struct(layers, packed)
    _ok(load_library().climber_history_encode(
        C.byref(cfg), C.byref(w), _ptr(tau), _ptr(x_hist), _ptr(scen), _ptr(beh), cache.handle,
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
        "climber_history_encode")


def climber_sumi_score(cfg: Config, layers, tau, cache: KVCache, x_cand, cand_off, m_total: int,
                       m_max: int, cand_scen, cand_beh, y_cand, workspace, stream=None, packed=None) -> None:
    w, keep = _weights_struct(layers, packed)
    _ok(load_library().climber_sumi_score(
        C.byref(cfg), C.byref(w), _ptr(tau), cache.handle, _ptr(x_cand), _ptr(cand_off), m_total,
        m_max, _ptr(cand_scen), _ptr(cand_beh), _ptr(y_cand), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)), "climber_sumi_score")


STATIC_SCRATCH_BYTES = 32 << 20


def climber_sumi_score_static(cfg: Config, layers, tau, cache: KVCache, x_cand, cand_off, m_total: int,
                              m_max: int, cand_scen, cand_beh, y_cand, packed, stream=None) -> None:
    """climber_sumi_score with the scratch in the library's fixed per-GPU array (allocates nothing)."""
    w, keep = _weights_struct(layers if layers is not None else [], packed)
    w.n_layers = cfg.n_layers
    _ok(load_library().climber_sumi_score_static(
        C.byref(cfg), C.byref(w), _ptr(tau), cache.handle, _ptr(x_cand), _ptr(cand_off), m_total,
        m_max, _ptr(cand_scen), _ptr(cand_beh), _ptr(y_cand), _stream(stream)),
        "climber_sumi_score_static")


def rel_bias(pos_table, time_table, hist_pos, hist_ts, cand_pos=None, cand_ts=None) -> RelBias:
    """climber_rel_bias from device tensors: tables [n_scen, n_beh, H, n_pos] / [..., n_time] fp32."""
    rb = RelBias(_ptr(pos_table), _ptr(time_table), int(pos_table.shape[-1]), int(time_table.shape[-1]),
                 _ptr(hist_pos), _ptr(hist_ts), _ptr(cand_pos), _ptr(cand_ts))
    rb._keep = (pos_table, time_table, hist_pos, hist_ts, cand_pos, cand_ts)
    return rb


def climber_attn_history_bias(cfg: Config, tau_layer, q, k, v, scen, beh, cache: KVCache, layer: int,
                              o_hist, bias: RelBias, stream=None) -> None:
    code = (_native or _load_native(load_library())).attn_history_bias(cfg, tau_layer, q, k, v, scen, beh, cache.handle, layer, o_hist, bias, stream)
    if code is None:
        code = load_library().climber_attn_history_bias(C.byref(cfg), _ptr(tau_layer), _ptr(q), _ptr(k), _ptr(v), _ptr(scen), _ptr(beh),
                                                        cache.handle, layer, _ptr(o_hist), C.byref(bias), _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_history_bias")


def climber_attn_sumi_bias(cfg: Config, tau_layer, cache: KVCache, layer: int, q_c, k_c, v_c, cand_off,
                           m_total: int, m_max: int, cand_scen, cand_beh, o_c, bias: RelBias,
                           stream=None) -> None:
    code = (_native or _load_native(load_library())).attn_sumi_bias(cfg, tau_layer, cache.handle, layer, q_c, k_c, v_c, cand_off, m_total, m_max,
                                                                    cand_scen, cand_beh, o_c, bias, stream)
    if code is None:
        code = load_library().climber_attn_sumi_bias(C.byref(cfg), _ptr(tau_layer), cache.handle, layer, _ptr(q_c), _ptr(k_c), _ptr(v_c),
                                                     _ptr(cand_off), m_total, m_max, _ptr(cand_scen), _ptr(cand_beh), _ptr(o_c), C.byref(bias),
                                                     _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_sumi_bias")


def climber_sumi_forward(cfg: Config, layers, tau, x_hist, scen, beh, x_cand, cand_off, m_total: int,
                         m_max: int, cand_scen, cand_beh, scratch_cache: KVCache, y_hist, y_cand, workspace,
                         stream=None, packed=None) -> None:
    """Training-side packed forward: histories and candidates together, no cache kept."""
    w, keep = _weights_struct(layers, packed)
    _ok(load_library().climber_sumi_forward(
        C.byref(cfg), C.byref(w), _ptr(tau), _ptr(x_hist), _ptr(scen), _ptr(beh), _ptr(x_cand),
        _ptr(cand_off), m_total, m_max, _ptr(cand_scen), _ptr(cand_beh), scratch_cache.handle,
        _ptr(y_hist), _ptr(y_cand), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)), "climber_sumi_forward")


def climber_bgf_workspace_bytes(cfg: Config, n_blocks: int, d_gate: int, m_total: int) -> int:
    return int(load_library().climber_bgf_workspace_bytes(C.byref(cfg), n_blocks, d_gate, m_total))


def climber_bgf_score(cfg: Config, atl_layer, w_down, w_up, w_head, tau_scen, b_head: float, n_blocks: int,
                      d_gate: int, e, cand_scen, m_total: int, y, score, workspace, stream=None) -> None:
    """Bit-wise gating fusion (Eq. (4)) + linear head over the candidates' block outputs e."""
    w = BgfWeights(_layer_struct(atl_layer), _ptr(w_down), _ptr(w_up), _ptr(w_head), _ptr(tau_scen), b_head,
                   n_blocks, d_gate)
    _ok(load_library().climber_bgf_score(C.byref(cfg), C.byref(w), _ptr(e), _ptr(cand_scen), m_total, _ptr(y),
                                         _ptr(score), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                         _stream(stream)), "climber_bgf_score")


def paged_kv(k, v, page_table, len, max_len: int, mass=None, stamp=None) -> PagedKV:
    """climber_paged_kv from contiguous device tensors: k, v [n_pages, n_kv_heads, page_size, d_head]; page_table int32 [n_seqs, table_ld];
    len int32 [n_seqs]; mass fp32, stamp int32 [n_pages, page_size]."""
    for t in (k, v, page_table, len, mass, stamp):
        if t is not None and not t.is_contiguous():
            raise ValueError("a paged cache is described by contiguous tensors")
    n_pages, n_kv_heads, page_size, d_head = k.shape
    n_seqs, table_ld = page_table.shape
    if v.shape != k.shape or len.numel() != n_seqs or any(t is not None and t.numel() != n_pages * page_size for t in (mass, stamp)):
        raise ValueError("k, v, page_table, len, mass and stamp are not of one cache")
    kinds = [str(t.dtype)[6:] for t in (k, v, page_table, len, mass, stamp) if t is not None]  # (without "torch.")
    if kinds != [kinds[0]] * 2 + ["int32"] * 2 + ["float32"] * (mass is not None) + ["int32"] * (stamp is not None) or \
            kinds[0] not in ("bfloat16", "float32"):
        raise ValueError("k, v are bfloat16 or float32, page_table, len and stamp int32, mass float32")
    if any(t is not None and t.device != k.device for t in (v, page_table, len, mass, stamp)):
        raise ValueError("k, v, page_table, len, mass and stamp are not on one device")
    kv = PagedKV(_ptr(k), _ptr(v), _ptr(mass), _ptr(stamp), _ptr(page_table), _ptr(len), n_pages, page_size, n_kv_heads, n_seqs, table_ld, max_len,
                 d_head, k.element_size())
    kv._keep = (k, v, mass, stamp, page_table, len)
    if k.is_cuda:
        kv._device = k.device.index
    elif not all(t is None or t.is_pinned() for t in kv._keep):
        kv._device = -1
    return kv


def _on_device(kv: PagedKV, stream) -> None:
    """A call without a stream goes to the current device's, a call with one to its device: that has to be the cache's."""
    at = kv._device
    if at == -1:
        raise ValueError("the paged cache is in host memory that no kernel can reach")
    if at is None or isinstance(stream, int):
        return
    import torch
    if at != (torch.cuda.current_device() if stream is None else getattr(stream, "device_index", at)):
        raise ValueError("the paged cache is on another device than the stream")


def _there(desc, *tensors) -> None:
    """What a call is given besides the described tensors lies on their device."""
    at = desc._device
    if at is not None and any(t is not None and not isinstance(t, int) and t.get_device() != at for t in tensors):
        raise ValueError("the call's tensors are not on the device of what it works on")


def climber_paged_workspace_bytes(cfg: Config, kv: PagedKV, m_total: int, m_max: int) -> int:
    return int(load_library().climber_paged_workspace_bytes(C.byref(cfg), C.byref(kv), m_total, m_max))


def _pitch(t, width: int) -> int:
    """Elements from one row to the next: of a tensor its first stride (its other dimensions lie one behind the other), of a pointer `width`."""
    if t is None or isinstance(t, int):
        return width
    shape, stride = t.shape, t.stride()
    inner = 1
    for n, st in zip(reversed(shape[1:]), reversed(stride[1:])):
        if n != 1 and st != inner:
            raise ValueError("the elements of a row have to be contiguous")
        inner *= n
    return stride[0] if shape[0] > 1 else max(width, inner)


def _same_pitch(k, v, width: int) -> int:
    ld = _pitch(k, width)
    if v is not None and not isinstance(v, int) and v.shape[0] > 1 and _pitch(v, width) != ld:
        raise ValueError("k and v have different row pitches")
    return ld


def climber_attn_history_paged(cfg: Config, tau_layer, kv: PagedKV, q, k, v, off, m_total: int, m_max: int, scen, beh, stamp, o,
                               workspace, stream=None) -> None:
    """Append a chunk of new behaviours to the paged cache and attend from them.  q, k, v, o: row r is [r] of the tensor (row pitches are
    taken from it, so that columns of one projection's output can be passed as they are)."""
    _on_device(kv, stream)
    code = (_native or _load_native(load_library())).attn_history_paged(cfg, tau_layer, kv, q, k, v, off, m_total, m_max, scen, beh, stamp, o,
                                                                        workspace, stream)
    if code is None:
        d, dk = cfg.d_model, kv.n_kv_heads * cfg.d_head
        code = load_library().climber_attn_history_paged(
            C.byref(cfg), _ptr(tau_layer), C.byref(kv), _ptr(q), _pitch(q, d), _ptr(k), _ptr(v), _same_pitch(k, v, dk), _ptr(off), m_total, m_max,
            _ptr(scen), _ptr(beh), _ptr(stamp), _ptr(o), _pitch(o, d), _ptr(workspace), _nbytes(workspace), _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_history_paged")


def climber_attn_sumi_paged(cfg: Config, tau_layer, kv: PagedKV, q_c, k_c, v_c, cand_off, m_total: int, m_max: int, cand_scen, cand_beh,
                            o_c, workspace, stream=None) -> None:
    """Candidates against the paged cache (rows as in climber_attn_history_paged)."""
    _on_device(kv, stream)
    code = (_native or _load_native(load_library())).attn_sumi_paged(cfg, tau_layer, kv, q_c, k_c, v_c, cand_off, m_total, m_max, cand_scen,
                                                                     cand_beh, o_c, workspace, stream)
    if code is None:
        d, dk = cfg.d_model, kv.n_kv_heads * cfg.d_head
        code = load_library().climber_attn_sumi_paged(
            C.byref(cfg), _ptr(tau_layer), C.byref(kv), _ptr(q_c), _pitch(q_c, d), _ptr(k_c), _ptr(v_c), _same_pitch(k_c, v_c, dk),
            _ptr(cand_off), m_total, m_max, _ptr(cand_scen), _ptr(cand_beh), _ptr(o_c), _pitch(o_c, d), _ptr(workspace), _nbytes(workspace),
            _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_sumi_paged")


def climber_paged_evict(cfg: Config, kv: PagedKV, rank, budget, keep_from, len_out, src, workspace, stream=None) -> None:
    """Cut every sequence of the paged cache to its budget, least weight first."""
    _on_device(kv, stream)
    code = (_native or _load_native(load_library())).paged_evict(cfg, kv, rank, budget, keep_from, len_out, src, workspace, stream)
    if code is None:
        code = load_library().climber_paged_evict(C.byref(cfg), C.byref(kv), _ptr(rank), _ptr(budget), _ptr(keep_from), _ptr(len_out), _ptr(src),
                                                  _ptr(workspace), _nbytes(workspace), _stream(stream))
    if code:
        raise ClimberError(code, "climber_paged_evict")


def climber_check_paged(cfg: Config, kv: PagedKV, off, m_total: int, m_max: int, appends: bool, status, stream=None) -> None:
    """Device-side check of page numbers / lengths / offsets; ORs BAD_* bits into status (int32 tensor)."""
    _on_device(kv, stream)
    _ok(load_library().climber_check_paged(C.byref(cfg), C.byref(kv), _ptr(off), m_total, m_max, int(appends), _ptr(status), _stream(stream)),
        "climber_check_paged")


def paged_kv8(k, v, k_scale, v_scale, page_table, len, max_len: int, stamp=None) -> PagedKV8:
    """climber_paged_kv8 from contiguous device tensors: k, v float8_e4m3fn or uint8 [n_pages, n_kv_heads, page_size, d_head]; k_scale, v_scale uint8
    (or float8_e8m0fnu) [n_pages, n_kv_heads, page_size / 16]; the others as in paged_kv."""
    tensors = [t for t in (k, v, k_scale, v_scale, page_table, len, stamp) if t is not None]
    for t in tensors:
        if not t.is_contiguous():
            raise ValueError("a paged cache is described by contiguous tensors")
    n_pages, n_kv_heads, page_size, d_head = k.shape
    n_seqs, table_ld = page_table.shape
    blocks = (n_pages, n_kv_heads, page_size // 16)
    if v.shape != k.shape or tuple(k_scale.shape) != blocks or tuple(v_scale.shape) != blocks or len.numel() != n_seqs or \
            (stamp is not None and stamp.numel() != n_pages * page_size):
        raise ValueError("k, v, k_scale, v_scale, page_table, len and stamp are not of one cache")
    kinds = [str(t.dtype)[6:] for t in tensors]  # (without "torch.")
    if any(x not in ("float8_e4m3fn", "uint8") for x in kinds[:2]) or any(x not in ("uint8", "float8_e8m0fnu") for x in kinds[2:4]) or \
            any(x != "int32" for x in kinds[4:]):
        raise ValueError("k, v are float8_e4m3fn or uint8, k_scale and v_scale uint8 or float8_e8m0fnu, page_table, len and stamp int32")
    if any(t.device != k.device for t in tensors):
        raise ValueError("k, v, k_scale, v_scale, page_table, len and stamp are not on one device")
    kv = PagedKV8(PagedKV(_ptr(k), _ptr(v), None, _ptr(stamp), _ptr(page_table), _ptr(len), n_pages, page_size, n_kv_heads, n_seqs, table_ld, max_len,
                          d_head, 1), _ptr(k_scale), _ptr(v_scale))
    kv._keep = tensors
    if k.is_cuda:
        kv._device = k.device.index
    elif not all(t.is_pinned() for t in tensors):
        kv._device = -1
    return kv


def climber_paged8_workspace_bytes(cfg: Config, kv8: PagedKV8, m_total: int, m_max: int) -> int:
    return int(load_library().climber_paged8_workspace_bytes(C.byref(cfg), C.byref(kv8), m_total, m_max))


def _read8(cfg: Config, kv8: PagedKV8, m_total: int, tau, off, ids, **rows) -> None:
    """What a call reads of its tensors is there, and of its type (where the cache is described by tensors on a device, and there are rows)."""
    if kv8._device is None or m_total <= 0:
        return
    _ints("float32", tau_layer=(tau, cfg.n_scen * cfg.n_beh))
    _ints(off=(off, kv8.kv.n_seqs + 1), **{n: (t, m_total) for n, t in zip(("scen", "beh", "stamp"), ids)})
    for name, (t, wide) in rows.items():
        if t is not None and not isinstance(t, int) and \
                (str(t.dtype) != "torch.bfloat16" or t.shape[0] < m_total or t.numel() < t.shape[0] * wide):
            raise ValueError(f"{name} is a bfloat16 tensor of {m_total} rows of {wide} elements or more")


def climber_attn_history_paged8(cfg: Config, tau_layer, kv8: PagedKV8, q, k, v, off, m_total: int, m_max: int, scen, beh, stamp, o,
                                workspace, stream=None) -> None:
    """climber_attn_history_paged on a cache in 8 bits.  Tensors of other types than the call reads (rows bfloat16, off, ids and stamps int32, temperatures
    float32), or with less in them, are a ValueError."""
    _on_device(kv8, stream)
    code = (_native or _load_native(load_library())).attn_history_paged8(cfg, tau_layer, kv8, q, k, v, off, m_total, m_max, scen, beh, stamp, o,
                                                                         workspace, stream, kv8._device)
    if code is None:
        _there(kv8, tau_layer, q, k, v, off, scen, beh, stamp, o, workspace)
        d, dk = cfg.d_model, kv8.kv.n_kv_heads * cfg.d_head
        _read8(cfg, kv8, m_total, tau_layer, off, (scen, beh, stamp), q=(q, d), k=(k, dk), v=(v, dk), o=(o, d))
        code = load_library().climber_attn_history_paged8(
            C.byref(cfg), _ptr(tau_layer), C.byref(kv8), _ptr(q), _pitch(q, d), _ptr(k), _ptr(v), _same_pitch(k, v, dk), _ptr(off), m_total, m_max,
            _ptr(scen), _ptr(beh), _ptr(stamp), _ptr(o), _pitch(o, d), _ptr(workspace), _nbytes(workspace), _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_history_paged8")


def climber_attn_sumi_paged8(cfg: Config, tau_layer, kv8: PagedKV8, q_c, k_c, v_c, cand_off, m_total: int, m_max: int, cand_scen, cand_beh,
                             o_c, workspace, stream=None) -> None:
    """climber_attn_sumi_paged on a cache in 8 bits.  Tensors as in climber_attn_history_paged8."""
    _on_device(kv8, stream)
    code = (_native or _load_native(load_library())).attn_sumi_paged8(cfg, tau_layer, kv8, q_c, k_c, v_c, cand_off, m_total, m_max, cand_scen,
                                                                      cand_beh, o_c, workspace, stream, kv8._device)
    if code is None:
        _there(kv8, tau_layer, q_c, k_c, v_c, cand_off, cand_scen, cand_beh, o_c, workspace)
        d, dk = cfg.d_model, kv8.kv.n_kv_heads * cfg.d_head
        _read8(cfg, kv8, m_total, tau_layer, cand_off, (cand_scen, cand_beh), q_c=(q_c, d), k_c=(k_c, dk), v_c=(v_c, dk), o_c=(o_c, d))
        code = load_library().climber_attn_sumi_paged8(
            C.byref(cfg), _ptr(tau_layer), C.byref(kv8), _ptr(q_c), _pitch(q_c, d), _ptr(k_c), _ptr(v_c), _same_pitch(k_c, v_c, dk),
            _ptr(cand_off), m_total, m_max, _ptr(cand_scen), _ptr(cand_beh), _ptr(o_c), _pitch(o_c, d), _ptr(workspace), _nbytes(workspace),
            _stream(stream))
    if code:
        raise ClimberError(code, "climber_attn_sumi_paged8")


def page_pool(refs, page_table, held, len, page_size: int) -> PagePool:
    """climber_page_pool from contiguous int32 device tensors: refs [n_pages], page_table [n_seqs, table_ld], held, len [n_seqs]."""
    tensors = (refs, page_table, held, len)
    if any(not t.is_contiguous() or str(t.dtype) != "torch.int32" for t in tensors):
        raise ValueError("refs, page_table, held and len are contiguous tensors of int32")
    n_seqs, table_ld = page_table.shape
    if held.numel() != n_seqs or len.numel() != n_seqs:
        raise ValueError("page_table, held and len are not of one pool")
    if any(t.device != refs.device for t in tensors):
        raise ValueError("refs, page_table, held and len are not on one device")
    pool = PagePool(*(_ptr(t) for t in tensors), refs.numel(), page_size, n_seqs, table_ld)
    pool._keep = tensors
    if refs.is_cuda:
        pool._device = refs.device.index
    elif not all(t.is_pinned() for t in tensors):
        pool._device = -1
    return pool


def climber_pages_workspace_bytes(pool: PagePool) -> int:
    return int(load_library().climber_pages_workspace_bytes(C.byref(pool)))


def _ints(kind: str = "int32", **least) -> None:
    """name=(tensor, elements of the type that it has at least)"""
    for name, (t, n) in least.items():
        if t is not None and not isinstance(t, int) and (str(t.dtype) != "torch." + kind or not t.is_contiguous() or t.numel() < n):
            raise ValueError(f"{name} is a contiguous {kind} tensor of {n} or more")


def _room(copies, most: int) -> int:
    """Copies are read no further than there are any."""
    if copies is None or isinstance(copies, int):
        return most
    if not copies.is_contiguous():
        raise ValueError("copies are contiguous")
    return min(most, copies.numel() // 3)


def _copies(copies, counts):
    """An empty tensor has no address: one that there is, and of which nothing is read, in its place."""
    if copies is None or isinstance(copies, int) or copies.numel() > 0:
        return copies
    _ints(copies=(copies, 0))
    return counts


def climber_pages_fork(pool: PagePool, parent, keep, status, workspace, stream=None) -> None:
    """Sequence b becomes what sequence parent[b] was (below 0: empty), up to its first keep[b] tokens; pages are shared, and with keep no row holds
    more of them than its tokens need."""
    _on_device(pool, stream)
    code = (_native or _load_native(load_library())).pages_fork(pool, parent, keep, status, workspace, stream, pool._device)
    if code is None:
        _there(pool, parent, keep, status, workspace)
        _ints(parent=(parent, pool.n_seqs), keep=(keep, pool.n_seqs), status=(status, 1))
        code = load_library().climber_pages_fork(C.byref(pool), _ptr(parent), _ptr(keep), _ptr(status), _ptr(workspace), _nbytes(workspace),
                                                 _stream(stream))
    if code:
        raise ClimberError(code, "climber_pages_fork")


def climber_pages_extend(pool: PagePool, rows, copies, counts, status, workspace, stream=None) -> None:
    """Pages for rows[b] more tokens of each sequence; shared pages that they go into are replaced, and copies says by which."""
    _on_device(pool, stream)
    code = (_native or _load_native(load_library())).pages_extend(pool, rows, copies, counts, status, workspace, stream, pool._device)
    if code is None:
        _there(pool, rows, copies, counts, status, workspace)
        _ints(rows=(rows, pool.n_seqs), copies=(copies, 3 * pool.n_seqs), counts=(counts, 2), status=(status, 1))
        code = load_library().climber_pages_extend(C.byref(pool), _ptr(rows), _ptr(copies), _ptr(counts), _ptr(status), _ptr(workspace),
                                                   _nbytes(workspace), _stream(stream))
    if code:
        raise ClimberError(code, "climber_pages_extend")


def climber_pages_compact(pool: PagePool, copies, counts, status, workspace, stream=None) -> None:
    """The pages in use move to the front of the pool; copies says which went where."""
    _on_device(pool, stream)
    code = (_native or _load_native(load_library())).pages_compact(pool, copies, counts, status, workspace, stream, pool._device)
    if code is None:
        _there(pool, copies, counts, status, workspace)
        _ints(copies=(copies, pool.n_pages // 2 * 3), counts=(counts, 2), status=(status, 1))
        code = load_library().climber_pages_compact(C.byref(pool), _ptr(copies), _ptr(counts), _ptr(status), _ptr(workspace), _nbytes(workspace),
                                                    _stream(stream))
    if code:
        raise ClimberError(code, "climber_pages_compact")


def climber_paged_copy(cfg: Config, kv: PagedKV, copies, counts, max_copies: int, stream=None) -> None:
    """What climber_pages_extend or climber_pages_compact has left to copy, in one paged cache."""
    _on_device(kv, stream)
    max_copies = _room(copies, max_copies)
    if max_copies == 0:
        copies = _copies(copies, counts)
    code = (_native or _load_native(load_library())).paged_copy(cfg, kv, copies, counts, max_copies, stream, kv._device)
    if code is None:
        _there(kv, copies, counts)
        _ints(copies=(copies, 3 * max_copies), counts=(counts, 1))
        code = load_library().climber_paged_copy(C.byref(cfg), C.byref(kv), _ptr(copies), _ptr(counts), max_copies, _stream(stream))
    if code:
        raise ClimberError(code, "climber_paged_copy")


def climber_paged8_copy(cfg: Config, kv8: PagedKV8, copies, counts, max_copies: int, stream=None) -> None:
    """climber_paged_copy in a cache in 8 bits."""
    _on_device(kv8, stream)
    max_copies = _room(copies, max_copies)
    if max_copies == 0:
        copies = _copies(copies, counts)
    code = (_native or _load_native(load_library())).paged8_copy(cfg, kv8, copies, counts, max_copies, stream, kv8._device)
    if code is None:
        _there(kv8, copies, counts)
        _ints(copies=(copies, 3 * max_copies), counts=(counts, 1))
        code = load_library().climber_paged8_copy(C.byref(cfg), C.byref(kv8), _ptr(copies), _ptr(counts), max_copies, _stream(stream))
    if code:
        raise ClimberError(code, "climber_paged8_copy")


ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3


def climber_rotary_frequencies(rot_dims: int, base: float = 10000.0, kind: int = ROTARY_PLAIN, factor: float = 1.0, made_for: float = 0.0,
                               fast: float = 32.0, slow: float = 1.0):
    """(radians per position of each pair, what turned values are multiplied by)."""
    freq, scale = (C.c_double * max(1, rot_dims // 2))(), C.c_float()
    _ok(load_library().climber_rotary_frequencies(rot_dims, base, kind, factor, made_for, fast, slow, freq, C.byref(scale)),
        "climber_rotary_frequencies")
    return list(freq), scale.value


def rotary(freq, rot_dims: int, interleaved: bool = False, scale: float = 1.0, inverse: bool = False) -> RotaryPlan:
    """climber_rotary_plan from a float64 device tensor of rot_dims / 2 frequencies."""
    if str(freq.dtype) != "torch.float64" or not freq.is_contiguous() or freq.numel() != rot_dims // 2:
        raise ValueError("freq is a contiguous float64 tensor of rot_dims / 2 elements")
    plan = RotaryPlan(_ptr(freq), rot_dims, int(interleaved), int(inverse), scale)
    plan._keep = freq
    plan._device = freq.device.index if freq.is_cuda else None if freq.is_pinned() else -1
    return plan


def climber_rotary(cfg: Config, rot: RotaryPlan, pos, n_kv_heads: int, q, k, q_out, k_out, stream=None) -> None:
    """Turn q and k rows by their positions (row r is [r] of the tensors, as many rows as q has; row pitches are taken from them)."""
    _on_device(rot, stream)
    code = (_native or _load_native(load_library())).rotary(cfg, rot, pos, n_kv_heads, q, k, q_out, k_out, stream, rot._device)
    if code is None:
        _there(rot, pos, q, q_out, *((k, k_out) if n_kv_heads else ()))
        if pos.numel() != q.shape[0] or str(pos.dtype) != "torch.int32" or not pos.is_contiguous():
            raise ValueError("pos is a contiguous int32 tensor with a position for each row")
        m, d, dk = q.shape[0], cfg.d_model, n_kv_heads * cfg.d_head
        for t, wide in ((q, d), (q_out, d)) + (((k, dk), (k_out, dk)) if n_kv_heads else ()):
            if t.shape[0] != m or t.numel() != m * wide:
                raise ValueError("q, k, q_out and k_out have other rows")
            if str(t.dtype) != ("torch.float32" if cfg.dtype == F32 else "torch.bfloat16"):
                raise ValueError("q, k, q_out and k_out are of the configuration's type")
        code = load_library().climber_rotary(C.byref(cfg), C.byref(rot), _ptr(pos), m, n_kv_heads, _ptr(q), _pitch(q, d), _ptr(k), _pitch(k, dk),
                                             _ptr(q_out), _pitch(q_out, d), _ptr(k_out), _pitch(k_out, dk), _stream(stream))
    if code:
        raise ClimberError(code, "climber_rotary")
