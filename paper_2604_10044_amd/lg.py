"""Python binding of liblg (the C ABI in include/lg.h and include/lg_paged.h): argument marshalling only.

Every function here has the name of the C entry point it calls and takes torch tensors (device
memory) in place of raw pointers; those of the paged cache check the tensors' types, sizes, layout and
device first, which the C side cannot see. Importing this module loads liblg.so and raises if it is
missing: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblg.so")

if not os.path.exists(LIB_PATH):
    raise ImportError("liblg.so is not built (run __graft_entry__.build() or "
                      "python -m paper_2604_10044_amd.build)")
_lib = ctypes.CDLL(LIB_PATH)

LG_F32, LG_BF16 = 0, 1
LG_ATTEND_STATUS_WAIT, LG_ATTEND_STATUS_WORKSPACE = 1, 2
# test hooks (include/lg_testing.h)
FORM_AUTO, FORM_PORTABLE, FORM_MERGE, FORM_ONE_LAUNCH = 0, 1, 2, 3
TEST_FORCE_HANDOVER, TEST_NO_WAIT, TEST_WHOLE_DIMS = 1, 2, 4
LG_MODE_FULL, LG_MODE_ALWAYS_ON, LG_MODE_P1_ONLY = 0, 1, 2
LG_POLICY_LOOPGUARD, LG_POLICY_H2O, LG_POLICY_STREAMING = 0, 1, 2
LG_ROPE_PLAIN, LG_ROPE_LINEAR, LG_ROPE_BASE, LG_ROPE_RAMP, LG_ROPE_BANDS = 0, 1, 2, 3, 4
STATUS = {0: "LG_OK", 1: "LG_ERR_NULL", 2: "LG_ERR_SHAPE", 3: "LG_ERR_UNSUPPORTED",
          4: "LG_ERR_PARAM", 5: "LG_ERR_WORKSPACE", 6: "LG_ERR_HIP", 7: "LG_ERR_ALIGN",
          8: "LG_ERR_TOO_LARGE"}
NOALLOC_SCRATCH_BYTES = 64 << 20   # LG_NOALLOC_SCRATCH_BYTES

PARAM_FIELDS = ["W", "K", "n_anchor", "t_min", "cooldown", "streak_min", "stall_min",
                "cr_interval", "nov_ngram", "nov_span", "rep_pmax", "rep_horizon",
                "rep_min_copies", "rep_min_len", "rep_debounce", "level_max", "retrigger_window",
                "recent_div", "sparse_div", "ttr_num", "ttr_den", "cr_num", "cr_den", "nov_num",
                "nov_den"]
STATE_FIELDS = ["streak", "stall", "rep", "n_int", "n_last", "level", "cr_valid", "cr_cost",
                "cr_m"]
DECISION_FIELDS = ["trigger", "warn", "votes", "stall_gate", "tailrep_gate", "n", "distinct",
                   "lz_cost", "novel", "nov_r", "period", "span_lo", "level", "n_int"]
ATTEND_ERROR_COL = 14  # lg_decision.attend_error (not a decision of the paper's rule)
HEADER_FIELDS = ["magic", "version", "batch", "n_q_heads", "n_kv_heads", "head_dim", "cap",
                 "dtype", "form", "split", "status", "few_rows"]
STATE_INTS = 528     # lg_guard_state is 528 int32 (16 fields + 512 tail runs)
DECISION_INTS = 16   # lg_decision is 16 int32


class LayerCache(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("cap", ctypes.c_int32), ("dtype", ctypes.c_int), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("acc", ctypes.c_void_p)]


class GuardParams(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in PARAM_FIELDS] + [
        ("conf_threshold", ctypes.c_float), ("mode", ctypes.c_int32), ("policy", ctypes.c_int32)]

    def as_dict(self):
        d = {f: int(getattr(self, f)) for f in PARAM_FIELDS}
        d["conf_threshold"] = float(self.conf_threshold)
        d["mode"] = int(self.mode)
        d["policy"] = int(self.policy)
        return d


class PageMap(ctypes.Structure):
    """lg_page_map; made by page_map(), which keeps the tensors alive in `tensors`."""
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("table", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("len", ctypes.c_void_p), ("ref", ctypes.c_void_p)]


class PagedLayer(ctypes.Structure):
    """lg_paged_layer; made by paged_layer(), which keeps the tensors alive in `tensors`."""
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p)]


class RopeParams(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("theta", ctypes.c_double),
                ("factor", ctypes.c_double), ("original_context", ctypes.c_double),
                ("slow", ctypes.c_double), ("fast", ctypes.c_double)]


_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_lib.lg_guard_params_default.restype = GuardParams
_lib.lg_guard_params_default.argtypes = []
_lib.lg_status_string.restype = ctypes.c_char_p
_lib.lg_status_string.argtypes = [ctypes.c_int]
_lib.lg_state_bytes.restype = _sz
_lib.lg_decision_bytes.restype = _sz
_LP = ctypes.POINTER(LayerCache)
_lib.lg_decode_attend_workspace.restype = _sz
_lib.lg_decode_attend_workspace.argtypes = [_LP]
_lib.lg_decode_attend_workspace_init.restype = ctypes.c_int
_lib.lg_decode_attend_workspace_init.argtypes = [_LP, _vp, _sz, _vp]
_ATT = [_LP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz]
_lib.lg_decode_attend.restype = ctypes.c_int
_lib.lg_decode_attend.argtypes = _ATT + [_vp]
_lib.lg_decode_attend_noalloc.restype = ctypes.c_int
_lib.lg_decode_attend_noalloc.argtypes = _ATT[:-2] + [_i32, _vp]
_lib.lg_test_attend_workspace.restype = _sz
_lib.lg_test_attend_workspace.argtypes = [_LP, _i32, _i32]
_lib.lg_test_attend_workspace_init.restype = ctypes.c_int
_lib.lg_test_attend_workspace_init.argtypes = [_LP, _i32, _i32, _vp, _sz, _vp]
_lib.lg_test_decode_attend.restype = ctypes.c_int
_lib.lg_test_decode_attend.argtypes = _ATT + [_i32, _i32, _i32, _vp]
_lib.lg_detect_loop.restype = ctypes.c_int
_lib.lg_detect_loop.argtypes = [ctypes.POINTER(GuardParams), _i32, _vp, _i32, _vp, _vp, _vp, _vp,
                                _vp, _vp]
_lib.lg_prune_compact.restype = ctypes.c_int
_lib.lg_prune_compact.argtypes = [ctypes.POINTER(GuardParams), _i32, _i32, _i32,
                                  ctypes.POINTER(LayerCache), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _vp]
_lib.lg_detect_and_prune.restype = ctypes.c_int
_lib.lg_detect_and_prune.argtypes = [ctypes.POINTER(GuardParams), _i32, _vp, _i32, _vp, _vp, _vp,
                                     _vp, _vp, _i32, _i32, ctypes.POINTER(LayerCache), _vp, _vp,
                                     _vp, _vp, _vp, _vp, _vp]
_MP, _PP = ctypes.POINTER(PageMap), ctypes.POINTER(PagedLayer)
_lib.lg_page_workspace.restype = _sz
_lib.lg_page_workspace.argtypes = [_MP]
_lib.lg_page_reserve.restype = ctypes.c_int
_lib.lg_page_reserve.argtypes = [_MP, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lg_page_fork.restype = ctypes.c_int
_lib.lg_page_fork.argtypes = [_MP, _vp, _vp, _sz, _vp]
_lib.lg_page_compact.restype = ctypes.c_int
_lib.lg_page_compact.argtypes = [_MP, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lg_rope_frequencies.restype = ctypes.c_int
_lib.lg_rope_frequencies.argtypes = [ctypes.POINTER(RopeParams), _vp, ctypes.POINTER(ctypes.c_float)]
_lib.lg_rope_append.restype = ctypes.c_int
_lib.lg_rope_append.argtypes = [_PP, _MP, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i32, _i32, ctypes.c_float, _vp,
                                _vp, _vp, _i32, _vp]
_lib.lg_paged_attend_workspace.restype = _sz
_lib.lg_paged_attend_workspace.argtypes = [_PP, _MP, _i32, _i32]
_lib.lg_paged_attend.restype = ctypes.c_int
_lib.lg_paged_attend.argtypes = [_PP, _MP, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _sz,
                                 _vp]
_lib.lg_copy_bandwidth.restype = ctypes.c_int
_lib.lg_copy_bandwidth.argtypes = [_vp, _vp, _sz, _vp]


class LGError(RuntimeError):
    pass


def _check(status: int, what: str):
    if status != 0:
        raise LGError("%s: %s (%s)" % (what, STATUS.get(status, status),
                                       _lib.lg_status_string(status).decode()))


# An attention call passes a dozen tensors, and on the small layers the marshalling is as long as the
# kernel: the common cases come first, and the current stream is read as its handle (no Stream object).
def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    try:
        return x.data_ptr()
    except AttributeError:
        if isinstance(x, int):
            return x
        raise


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_raw_stream(torch.cuda.current_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def _stream_handle(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_handle)


def lg_guard_params_default() -> GuardParams:
    return _lib.lg_guard_params_default()


def lg_status_string(status: int) -> str:
    return _lib.lg_status_string(status).decode()


def lg_state_bytes() -> int:
    return int(_lib.lg_state_bytes())


def lg_decision_bytes() -> int:
    return int(_lib.lg_decision_bytes())


def lg_decode_attend_workspace(layer: "LayerCache") -> int:
    return int(_lib.lg_decode_attend_workspace(ctypes.byref(layer)))


def lg_decode_attend_workspace_init(layer: "LayerCache", workspace, stream=None):
    ws = workspace.numel() * workspace.element_size()
    _check(_lib.lg_decode_attend_workspace_init(ctypes.byref(layer), _ptr(workspace), ws,
                                                _stream(stream)), "lg_decode_attend_workspace_init")


def lg_test_attend_workspace(layer: "LayerCache", form: int, max_split: int = 0) -> int:
    return int(_lib.lg_test_attend_workspace(ctypes.byref(layer), form, max_split))


def lg_test_attend_workspace_init(layer: "LayerCache", form: int, max_split: int, workspace,
                                  stream=None):
    ws = workspace.numel() * workspace.element_size()
    _check(_lib.lg_test_attend_workspace_init(ctypes.byref(layer), form, max_split,
                                              _ptr(workspace), ws, _stream(stream)),
           "lg_test_attend_workspace_init")


def workspace_header(workspace) -> dict:
    """The lg_attend_workspace_header at the start of a workspace, read back to the host."""
    h = workspace[:64].cpu().numpy().view("<i4")
    return {f: int(h[i]) & 0xffffffff if f in ("magic", "version", "status") else int(h[i])
            for i, f in enumerate(HEADER_FIELDS)}


def layer_cache(k: torch.Tensor, v: torch.Tensor, acc: torch.Tensor, n_q_heads: int) -> LayerCache:
    """View of one layer's cache: k, v [B][Hkv][cap][D] (float32 or bfloat16), acc [B][Hkv][cap]."""
    B, Hkv, cap, D = k.shape
    dt = LG_BF16 if k.dtype == torch.bfloat16 else LG_F32
    return LayerCache(B, n_q_heads, Hkv, D, cap, dt, k.data_ptr(), v.data_ptr(), acc.data_ptr())


def lg_decode_attend(layer: LayerCache, q, k_new, v_new, out, pos, len_, t, suffix_w, lse,
                     suffix_mass, conf, workspace, stream=None):
    ws = workspace.numel() * workspace.element_size()
    _check(_lib.lg_decode_attend(ctypes.byref(layer), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                                 _ptr(pos), _ptr(len_), _ptr(t), _ptr(suffix_w), _ptr(lse),
                                 _ptr(suffix_mass), _ptr(conf), _ptr(workspace), ws,
                                 _stream(stream)), "lg_decode_attend")


def lg_decode_attend_noalloc(layer: LayerCache, q, k_new, v_new, out, pos, len_, t, suffix_w, lse,
                             suffix_mass, conf, reinit: int = 0, stream=None):
    _check(_lib.lg_decode_attend_noalloc(ctypes.byref(layer), _ptr(q), _ptr(k_new), _ptr(v_new),
                                         _ptr(out), _ptr(pos), _ptr(len_), _ptr(t),
                                         _ptr(suffix_w), _ptr(lse), _ptr(suffix_mass), _ptr(conf),
                                         int(reinit), _stream(stream)),
           "lg_decode_attend_noalloc")


def lg_test_decode_attend(layer: LayerCache, q, k_new, v_new, out, pos, len_, t, suffix_w, lse,
                          suffix_mass, conf, workspace, form: int, max_split: int = 0,
                          flags: int = 0, stream=None):
    ws = workspace.numel() * workspace.element_size()
    _check(_lib.lg_test_decode_attend(ctypes.byref(layer), _ptr(q), _ptr(k_new), _ptr(v_new),
                                      _ptr(out), _ptr(pos), _ptr(len_), _ptr(t), _ptr(suffix_w),
                                      _ptr(lse), _ptr(suffix_mass), _ptr(conf), _ptr(workspace),
                                      ws, form, max_split, flags, _stream(stream)),
           "lg_test_decode_attend")


def lg_detect_loop(params: GuardParams, tokens, ring: int, t, t0, conf, state, decision,
                   stream=None):
    batch = t.shape[0]
    _check(_lib.lg_detect_loop(ctypes.byref(params), batch, _ptr(tokens), ring, _ptr(t), _ptr(t0),
                               _ptr(conf), _ptr(state), _ptr(decision), _stream(stream)),
           "lg_detect_loop")


def lg_prune_compact(params: GuardParams, batch: int, cap: int, layers: Sequence[LayerCache],
                     pos, len_, budget, t_append, decision, keep_idx, new_len, stream=None):
    n = len(layers)
    arr = (LayerCache * max(1, n))(*layers) if n else None
    _check(_lib.lg_prune_compact(ctypes.byref(params), batch, cap, n, arr, _ptr(pos), _ptr(len_),
                                 _ptr(budget), _ptr(t_append), _ptr(decision), _ptr(keep_idx),
                                 _ptr(new_len), _stream(stream)), "lg_prune_compact")


def lg_detect_and_prune(params: GuardParams, tokens, ring: int, t, t0, conf, state, decision,
                        cap: int, layers: Sequence[LayerCache], pos, len_, budget, t_append,
                        keep_idx, new_len, stream=None):
    batch = t.shape[0]
    n = len(layers)
    arr = (LayerCache * max(1, n))(*layers) if n else None
    _check(_lib.lg_detect_and_prune(ctypes.byref(params), batch, _ptr(tokens), ring, _ptr(t),
                                    _ptr(t0), _ptr(conf), _ptr(state), _ptr(decision), cap, n,
                                    arr, _ptr(pos), _ptr(len_), _ptr(budget), _ptr(t_append),
                                    _ptr(keep_idx), _ptr(new_len), _stream(stream)),
           "lg_detect_and_prune")


def lg_copy_bandwidth(src, dst, nbytes: int, stream=None):
    _check(_lib.lg_copy_bandwidth(_ptr(src), _ptr(dst), nbytes, _stream(stream)),
           "lg_copy_bandwidth")


# ------------------------------------------------------------------------------------------------
# The paged cache (include/lg_paged.h).
# ------------------------------------------------------------------------------------------------
# A decode step makes these calls for every layer, and the small ones take the GPU less time than the host: one
# comparison a property, and no message before something is wrong.
def _need(x, dtype, n, device, what):
    """The address of a tensor that is dense, of this type, on this device and of at least n values."""
    if x.dtype is dtype and x.numel() >= n and x.is_contiguous() and x.get_device() == device:
        return x.data_ptr()
    raise LGError("%s: needs a contiguous %s tensor of %d values on device %d, got %s %s on %s" %
                  (what, dtype, n, device, x.dtype, tuple(x.shape), x.device))


def _on(device: int, stream, layer=None):
    """The stream of a paged call, which runs on the current device: the map's and the layer's."""
    if layer is not None and layer.device != device:
        raise LGError("the layer's pages are on device %d, the page map on device %d" % (layer.device, device))
    if torch.cuda.current_device() != device:
        raise LGError("the page map is on device %d, the current device is %d" %
                      (device, torch.cuda.current_device()))
    return _current_raw_stream(device) if stream is None else _stream(stream)


def _bytes(workspace, device, what):
    if workspace.get_device() != device or not workspace.is_contiguous():
        raise LGError("%s: needs a contiguous workspace on device %d" % (what, device))
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def page_map(table: torch.Tensor, pos: torch.Tensor, len_: torch.Tensor, ref: torch.Tensor,
             page_size: int) -> PageMap:
    """The map of a paged cache: int32 table [B][P], pos [B][P * page_size], len [B], ref [n_pages]."""
    B, P = table.shape
    dev = table.get_device()
    if dev < 0:
        raise LGError("page_map: needs device tensors")
    m = PageMap(B, P, ref.numel(), page_size, _need(table, torch.int32, B * P, dev, "table"),
                _need(pos, torch.int32, B * P * page_size, dev, "pos"),
                _need(len_, torch.int32, B, dev, "len"), _need(ref, torch.int32, 1, dev, "ref"))
    m.tensors, m.device = (table, pos, len_, ref), dev
    return m


def paged_layer(k: torch.Tensor, v: torch.Tensor, n_q_heads: int) -> PagedLayer:
    """View of one layer's pages: k, v [n_pages][Hkv][page_size][D] (float32 or bfloat16)."""
    n, Hkv, ps, D = k.shape
    if k.dtype not in (torch.float32, torch.bfloat16) or v.shape != k.shape:
        raise LGError("paged_layer: needs k and v of one shape, float32 or bfloat16")
    dev = k.get_device()
    if dev < 0:
        raise LGError("paged_layer: needs device tensors")
    l = PagedLayer(n, ps, n_q_heads, Hkv, D, LG_BF16 if k.dtype == torch.bfloat16 else LG_F32,
                   _need(k, k.dtype, 1, dev, "k"), _need(v, k.dtype, 1, dev, "v"))
    l.tensors, l.device, l.torch_dtype = (k, v), dev, k.dtype
    return l


def _layers(layers: Sequence[PagedLayer], device):
    """The views side by side, as the host array that the C side reads during the call."""
    for l in layers:
        if l.device != device:
            raise LGError("a layer's pages are on device %d, the page map on device %d" % (l.device, device))
    return b"".join(layers) or None


def lg_page_workspace(m: PageMap) -> int:
    return int(_lib.lg_page_workspace(ctypes.byref(m)))


def lg_page_reserve(m: PageMap, layers: Sequence[PagedLayer], q_start, t, base, workspace, stream=None):
    dev, B, i32 = m.device, m.batch, torch.int32
    stream = _on(dev, stream)
    ws, size = _bytes(workspace, dev, "workspace")
    _check(_lib.lg_page_reserve(ctypes.byref(m), len(layers), _layers(layers, dev),
                                _need(q_start, i32, B + 1, dev, "q_start"), _need(t, i32, B, dev, "t"),
                                _need(base, i32, B, dev, "base"), ws, size, stream),
           "lg_page_reserve")


def lg_page_fork(m: PageMap, parent, workspace, stream=None):
    stream = _on(m.device, stream)
    ws, size = _bytes(workspace, m.device, "workspace")
    _check(_lib.lg_page_fork(ctypes.byref(m), _need(parent, torch.int32, m.batch, m.device, "parent"),
                             ws, size, stream), "lg_page_fork")


def lg_page_compact(m: PageMap, layers: Sequence[PagedLayer], keep_idx, new_len, moved, workspace, stream=None):
    dev, B, i32 = m.device, m.batch, torch.int32
    stream = _on(dev, stream)
    ws, size = _bytes(workspace, dev, "workspace")
    _check(_lib.lg_page_compact(ctypes.byref(m), len(layers), _layers(layers, dev),
                                _need(keep_idx, i32, B * m.max_pages * m.page_size, dev, "keep_idx"),
                                _need(new_len, i32, B, dev, "new_len"), _need(moved, i32, B, dev, "moved"),
                                ws, size, stream), "lg_page_compact")


def lg_rope_frequencies(params: RopeParams):
    """(inv_freq, scale): the frequencies as a float32 tensor on the host and the factor of cos and sin."""
    inv = torch.zeros(max(1, params.rot_dim // 2), dtype=torch.float32)
    scale = ctypes.c_float()
    _check(_lib.lg_rope_frequencies(ctypes.byref(params), inv.data_ptr(), ctypes.byref(scale)),
           "lg_rope_frequencies")
    return inv, scale.value


def _rows(x, heads, D, dtype, device, what):
    """(pointer, row stride) of x [total][heads][D], whose rows may lie apart."""
    shape, stride = x.shape, x.stride()
    if x.dtype is dtype and len(shape) == 3 and shape[1] == heads and shape[2] == D and stride[2] == 1 and \
            (stride[1] == D or heads == 1) and x.get_device() == device:
        return x.data_ptr(), (stride[0] if shape[0] > 1 else heads * D)
    raise LGError("%s: needs a %s tensor [rows][%d][%d] on device %d with dense heads, got %s %s on %s" %
                  (what, dtype, heads, D, device, x.dtype, tuple(shape), x.device))


def lg_rope_append(layer: PagedLayer, m: PageMap, q, k, v, inv_freq, rot_dim: int, interleaved, scale: float,
                   q_out, q_start, base, stream=None):
    dev, D, dt, i32 = m.device, layer.head_dim, layer.torch_dtype, torch.int32
    stream = _on(dev, stream, layer)
    total = q.shape[0]
    qp, qs = _rows(q, layer.n_q_heads, D, dt, dev, "q")
    kp = vp = None
    ks = vs = 0
    if k is not None or v is not None:
        if k is None or v is None or k.shape[0] != total or v.shape[0] != total:
            raise LGError("lg_rope_append: needs k and v of as many rows as q, or neither")
        kp, ks = _rows(k, layer.n_kv_heads, D, dt, dev, "k")
        vp, vs = _rows(v, layer.n_kv_heads, D, dt, dev, "v")
    fp = None if rot_dim == 0 else _need(inv_freq, torch.float32, rot_dim // 2, dev, "inv_freq")
    _check(_lib.lg_rope_append(ctypes.byref(layer), ctypes.byref(m), qp, qs, kp, ks, vp, vs, fp, rot_dim,
                               int(bool(interleaved)), scale,
                               _need(q_out, dt, total * layer.n_q_heads * D, dev, "q_out"),
                               _need(q_start, i32, m.batch + 1, dev, "q_start"),
                               _need(base, i32, m.batch, dev, "base"), total, stream),
           "lg_rope_append")


def lg_paged_attend_workspace(layer: PagedLayer, m: PageMap, total: int, max_chunk: int) -> int:
    return int(_lib.lg_paged_attend_workspace(ctypes.byref(layer), ctypes.byref(m), total, max_chunk))


def lg_paged_attend(layer: PagedLayer, m: PageMap, q, out, q_start, base, max_chunk: int, window: int,
                    n_sink: int, suffix_w, lse, suffix_mass, conf, workspace, stream=None):
    dev, B, dt, i32, f32 = m.device, m.batch, layer.torch_dtype, torch.int32, torch.float32
    stream = _on(dev, stream, layer)
    total, n = q.shape[0], q.shape[0] * layer.n_q_heads
    ws, size = _bytes(workspace, dev, "workspace")
    _check(_lib.lg_paged_attend(
        ctypes.byref(layer), ctypes.byref(m), _need(q, dt, n * layer.head_dim, dev, "q"),
        _need(out, dt, n * layer.head_dim, dev, "out"), _need(q_start, i32, B + 1, dev, "q_start"),
        _need(base, i32, B, dev, "base"), total, max_chunk, window, n_sink,
        None if suffix_w is None else _need(suffix_w, i32, B, dev, "suffix_w"),
        _need(lse, f32, n, dev, "lse"),
        None if suffix_mass is None else _need(suffix_mass, f32, n, dev, "suffix_mass"),
        None if conf is None else _need(conf, f32, B, dev, "conf"), ws, size, stream),
        "lg_paged_attend")


def params_from_dict(d) -> GuardParams:
    p = lg_guard_params_default()
    for k, v in d.items():
        setattr(p, k, v)
    return p
