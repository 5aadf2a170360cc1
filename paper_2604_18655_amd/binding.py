"""ctypes binding of the headers in include/.  Tensors are torch CUDA(HIP) tensors used as plain
device buffers; work is enqueued on torch's current stream."""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmlora_w4.so")
_lib = None

Y_BF16, Y_FP32 = 0, 1

exported_symbols = (
    "mlora_strerror", "mlora_w4_blob_bytes", "mlora_w4_prepack", "mlora_w4_unpack",
    "mlora_group_rows", "mlora_w4_workspace_bytes", "mlora_w4_linear", "mlora_w4_layer_step",
    "mlora_w4_workspace_init", "mlora_w4_workspace_status", "mlora_w4_debug_spin_limit",
    "mlora_w4_layer_step_static", "mlora_w4_layer_step_plan", "mlora_w4_layer_step_block_rows",
    "mlora_w4_layer_step_waves_per_tile",
    "mlora_tree_attention_workspace_bytes", "mlora_tree_attention_plan", "mlora_tree_attention",
    "mlora_w4a8_workspace_bytes", "mlora_w4a8_layer_step",
    "mlora_w4_layer_step_fused", "mlora_rms_scale", "mlora_lora_int16_expand",
    "mlora_ds2d_rows", "mlora_ds2d_layout", "mlora_ds2d_workspace_bytes", "mlora_ds2d_late_drafts",
    "mlora_ds2d_step",
)
# of mlora_rope.h, mlora_stream_cache.h and mlora_logit_rules.h: what a decoding loop does around these
loop_symbols = (
    "mlora_rope_frequencies", "mlora_rope_tables", "mlora_rope_apply",
    "mlora_stream_cache_append", "mlora_stream_cache_compress",
    "mlora_attention_mass_workspace_bytes", "mlora_attention_mass_add",
    "mlora_logit_rules_apply",
)
# of mlora_page_cache.h, mlora_page_attention.h and mlora_beam.h: beam search on a paged cache of 8 bits
beam_symbols = (
    "mlora_page_cache_own_words", "mlora_page_cache_append", "mlora_page_cache_reorder", "mlora_page_cache_copy",
    "mlora_page_attention_workspace_bytes", "mlora_page_attention_plan", "mlora_page_attention",
    "mlora_beam_workspace_bytes", "mlora_beam_select",
)


class MloraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


class _ProjStruct(C.Structure):
    _fields_ = [("K", C.c_int32), ("N", C.c_int32), ("group", C.c_int32),
                ("w_blob", C.c_void_p), ("n_adapters", C.c_int32), ("rank", C.c_int32),
                ("lora_a", C.c_void_p), ("lora_b", C.c_void_p), ("alpha", C.c_float)]


class _Ds2dStruct(C.Structure):
    _fields_ = [("n_streams", C.c_int32), ("n_forecast", C.c_int32), ("depth", C.c_int32),
                ("branch", C.c_int32 * 8), ("next_depth", C.c_int32), ("next_branch", C.c_int32 * 8),
                ("vocab", C.c_int32), ("logits_dtype", C.c_int32)]


class _EpilogueStruct(C.Structure):
    _fields_ = [("row_scale", C.c_void_p), ("pair_op", C.c_int32), ("rope_cos", C.c_void_p),
                ("rope_sin", C.c_void_p), ("residual", C.c_void_p), ("sq_in", C.c_void_p),
                ("sq_parts", C.c_int32), ("sq_eps", C.c_float), ("sq_out", C.c_void_p)]


class _TreeAttnStruct(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("n_streams", C.c_int32), ("rows_per_stream", C.c_int32), ("scale", C.c_float),
                ("k_prefill", C.c_void_p), ("v_prefill", C.c_void_p), ("len_prefill", C.c_int32),
                ("k_fprefix", C.c_void_p), ("v_fprefix", C.c_void_p), ("len_fprefix", C.c_int32),
                ("k_stream", C.c_void_p), ("v_stream", C.c_void_p), ("cap_stream", C.c_int32),
                ("len_stream", C.c_void_p),
                ("k_new", C.c_void_p), ("v_new", C.c_void_p),
                ("parent", C.c_void_p), ("is_forecast", C.c_void_p)]


class _RopeStruct(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("theta", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("context", C.c_double)]


class _RopeRowsStruct(C.Structure):
    _fields_ = [("M", C.c_int32), ("rows_per_stream", C.c_int32), ("base", C.c_void_p), ("offset", C.c_void_p),
                ("quarter_turns", C.c_void_p)]


class _RopeTensorStruct(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("x_row", C.c_int64), ("x_head", C.c_int64),
                ("y_row", C.c_int64), ("y_head", C.c_int64), ("heads", C.c_int32), ("rotate", C.c_int32)]


class _StreamCacheStruct(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_streams", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("cap", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("mass", C.c_void_p), ("slot_pos", C.c_void_p), ("len", C.c_void_p), ("next_pos", C.c_void_p),
                ("tickets", C.c_void_p)]


class _AttentionMassStruct(C.Structure):
    _fields_ = [("cache", _StreamCacheStruct), ("n_q_heads", C.c_int32), ("rows_per_stream", C.c_int32),
                ("scale", C.c_float), ("k_prefill", C.c_void_p), ("mass_prefill", C.c_void_p),
                ("len_prefill", C.c_int32), ("decay", C.c_float)]


class _LogitRulesStruct(C.Structure):
    _fields_ = [("n_streams", C.c_int32), ("rows_per_stream", C.c_int32), ("tokens_per_stream", C.c_int32),
                ("vocab", C.c_int32), ("logits_dtype", C.c_int32), ("parent", C.c_void_p), ("counts", C.c_void_p),
                ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p),
                ("bias", C.c_void_p), ("bias_row", C.c_void_p), ("n_bias", C.c_int32), ("masks", C.c_void_p),
                ("mask_row", C.c_void_p), ("n_masks", C.c_int32)]


class _PageCacheStruct(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_streams", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("k_tail", C.c_void_p), ("v_tail", C.c_void_p),
                ("slot", C.c_void_p), ("len", C.c_void_p), ("table", C.c_void_p), ("refs", C.c_void_p), ("own", C.c_void_p)]


class _PageAttnStruct(C.Structure):
    _fields_ = [("cache", _PageCacheStruct), ("layer", C.c_int32), ("n_q_heads", C.c_int32), ("rows_per_stream", C.c_int32),
                ("scale", C.c_float), ("window", C.c_int32), ("sink", C.c_int32), ("k_new", C.c_void_p), ("v_new", C.c_void_p),
                ("parent", C.c_void_p)]


class _BeamStruct(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("n_beams", C.c_int32), ("vocab", C.c_int32), ("logits_dtype", C.c_int32),
                ("eos", C.c_int32), ("pad", C.c_int32), ("length_power", C.c_float)]


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libmlora_w4.so; raises if it is missing (there is no other implementation)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} not built: run __graft_entry__.build() "
                              "(hipcc --offload-arch=gfx950)")
        lib = C.CDLL(_LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        pp = C.POINTER(_ProjStruct)
        lib.mlora_strerror.restype = C.c_char_p
        lib.mlora_strerror.argtypes = [C.c_int]
        lib.mlora_w4_blob_bytes.restype = sz
        lib.mlora_w4_blob_bytes.argtypes = [i32, i32, i32]
        lib.mlora_w4_prepack.restype = C.c_int
        lib.mlora_w4_prepack.argtypes = [i32, i32, i32, vp, vp, vp, vp]
        lib.mlora_w4_unpack.restype = C.c_int
        lib.mlora_w4_unpack.argtypes = [pp, vp, vp, vp]
        lib.mlora_group_rows.restype = C.c_int
        lib.mlora_group_rows.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
        lib.mlora_w4_workspace_bytes.restype = sz
        lib.mlora_w4_workspace_bytes.argtypes = [pp, i32, i32]
        lib.mlora_w4_linear.restype = C.c_int
        lib.mlora_w4_linear.argtypes = [pp, vp, vp, i32, vp, i32, vp, sz, vp]
        lib.mlora_w4_layer_step.restype = C.c_int
        lib.mlora_w4_layer_step.argtypes = [pp, i32, C.POINTER(vp), C.POINTER(vp), vp, i32, i32,
                                            vp, sz, vp]
        lib.mlora_w4_layer_step_static.restype = C.c_int
        lib.mlora_w4_layer_step_static.argtypes = [pp, i32, C.POINTER(vp), C.POINTER(vp), vp, i32, i32, vp]
        lib.mlora_w4_workspace_init.restype = C.c_int
        lib.mlora_w4_workspace_init.argtypes = [vp, sz, vp]
        tp = C.POINTER(_TreeAttnStruct)
        lib.mlora_tree_attention_workspace_bytes.restype = sz
        lib.mlora_tree_attention_workspace_bytes.argtypes = [tp]
        lib.mlora_tree_attention_plan.restype = C.c_int
        lib.mlora_tree_attention_plan.argtypes = [tp, C.POINTER(i32)]
        lib.mlora_tree_attention.restype = C.c_int
        lib.mlora_tree_attention.argtypes = [tp, vp, vp, i32, vp, sz, vp]
        lib.mlora_w4a8_workspace_bytes.restype = sz
        lib.mlora_w4a8_workspace_bytes.argtypes = [pp, i32, i32]
        lib.mlora_w4a8_layer_step.restype = C.c_int
        lib.mlora_w4a8_layer_step.argtypes = [pp, i32, C.POINTER(vp), C.POINTER(C.c_float), C.POINTER(vp), vp,
                                              i32, i32, vp, sz, vp]
        lib.mlora_w4_layer_step_fused.restype = C.c_int
        lib.mlora_w4_layer_step_fused.argtypes = [pp, C.POINTER(_EpilogueStruct), i32, C.POINTER(vp), C.POINTER(vp),
                                                  vp, i32, i32, vp, sz, vp]
        lib.mlora_rms_scale.restype = C.c_int
        lib.mlora_rms_scale.argtypes = [vp, i32, i32, C.c_float, vp, vp]
        lib.mlora_lora_int16_expand.restype = C.c_int
        lib.mlora_lora_int16_expand.argtypes = [vp, vp, i32, i32, i32, i32, C.c_float, C.c_float, C.c_float,
                                                vp, vp, C.POINTER(C.c_float), vp]
        dp = C.POINTER(_Ds2dStruct)
        ip = C.POINTER(i32)
        lib.mlora_ds2d_rows.restype = C.c_int
        lib.mlora_ds2d_rows.argtypes = [ip, i32, i32, ip, ip]
        lib.mlora_ds2d_layout.restype = C.c_int
        lib.mlora_ds2d_layout.argtypes = [ip, i32, i32, ip, C.POINTER(C.c_uint8), ip]
        lib.mlora_ds2d_workspace_bytes.restype = sz
        lib.mlora_ds2d_workspace_bytes.argtypes = [dp]
        lib.mlora_ds2d_late_drafts.restype = i32
        lib.mlora_ds2d_late_drafts.argtypes = [dp]
        lib.mlora_ds2d_step.restype = C.c_int
        lib.mlora_ds2d_step.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        rp, cp = C.POINTER(_RopeStruct), C.POINTER(_StreamCacheStruct)
        lib.mlora_rope_frequencies.restype = C.c_int
        lib.mlora_rope_frequencies.argtypes = [rp, C.POINTER(C.c_double)]
        lib.mlora_rope_tables.restype = C.c_int
        lib.mlora_rope_tables.argtypes = [rp, C.POINTER(_RopeRowsStruct), vp, vp, vp]
        lib.mlora_rope_apply.restype = C.c_int
        lib.mlora_rope_apply.argtypes = [rp, C.POINTER(_RopeRowsStruct), C.POINTER(_RopeTensorStruct), i32, i32, i32, vp]
        lib.mlora_stream_cache_append.restype = C.c_int
        lib.mlora_stream_cache_append.argtypes = [cp, vp, vp, i32, vp, i32, i32, i32, i32, vp]
        lib.mlora_stream_cache_compress.restype = C.c_int
        lib.mlora_stream_cache_compress.argtypes = [cp, cp, vp, i32, i32, i32, vp]
        mp = C.POINTER(_AttentionMassStruct)
        lib.mlora_attention_mass_workspace_bytes.restype = sz
        lib.mlora_attention_mass_workspace_bytes.argtypes = [mp, i32]
        lib.mlora_attention_mass_add.restype = C.c_int
        lib.mlora_attention_mass_add.argtypes = [mp, vp, vp, i32, vp, sz, vp]
        lib.mlora_logit_rules_apply.restype = C.c_int
        lib.mlora_logit_rules_apply.argtypes = [C.POINTER(_LogitRulesStruct), vp, vp, vp, i32, vp, vp]
        gp, ap, bp = C.POINTER(_PageCacheStruct), C.POINTER(_PageAttnStruct), C.POINTER(_BeamStruct)
        lib.mlora_page_cache_own_words.restype = sz
        lib.mlora_page_cache_own_words.argtypes = [i32, i32]
        lib.mlora_page_cache_append.restype = C.c_int
        lib.mlora_page_cache_append.argtypes = [gp, vp, vp, i32, vp, i32, vp, vp]
        lib.mlora_page_cache_reorder.restype = C.c_int
        lib.mlora_page_cache_reorder.argtypes = [gp, vp, i32, i32, vp]
        lib.mlora_page_cache_copy.restype = C.c_int
        lib.mlora_page_cache_copy.argtypes = [gp, gp, vp, vp, vp]
        lib.mlora_page_attention_workspace_bytes.restype = sz
        lib.mlora_page_attention_workspace_bytes.argtypes = [ap]
        lib.mlora_page_attention_plan.restype = C.c_int
        lib.mlora_page_attention_plan.argtypes = [ap, C.POINTER(i32)]
        lib.mlora_page_attention.restype = C.c_int
        lib.mlora_page_attention.argtypes = [ap, vp, vp, i32, vp, sz, vp]
        lib.mlora_beam_workspace_bytes.restype = sz
        lib.mlora_beam_workspace_bytes.argtypes = [bp]
        lib.mlora_beam_select.restype = C.c_int
        lib.mlora_beam_select.argtypes = [bp] + [vp] * 10 + [sz, vp]
        lib.mlora_w4_workspace_status.restype = C.c_int
        lib.mlora_w4_workspace_status.argtypes = [vp, C.POINTER(i32), vp]
        lib.mlora_w4_debug_spin_limit.restype = i32
        lib.mlora_w4_debug_spin_limit.argtypes = [i32]
        _lib = lib
    return _lib


def strerror(status: int) -> str:
    return load_library().mlora_strerror(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise MloraError(status, where)


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


_raw_stream = _device = None


class _PublicStream:
    """The two calls of _stream() by torch's public ones, for a torch without the private pair."""

    @staticmethod
    def _cuda_getDevice() -> int:
        import torch
        return torch.cuda.current_device()

    @staticmethod
    def _cuda_getCurrentRawStream(device: int) -> int:
        import torch
        return int(torch.cuda.current_stream(device).cuda_stream)


def _stream() -> int:
    """torch's current stream on the current device, without the Python object around it: 2.9 us of a
    call's 8.9 us of host time, where its kernel takes 6.0 (256 x 256 at 8 rows)."""
    global _raw_stream, _device
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()                      # initialises the device, or says why it cannot
        both = hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice")
        calls = torch._C if both else _PublicStream
        _device, _raw_stream = calls._cuda_getDevice, calls._cuda_getCurrentRawStream
    return _raw_stream(_device())


def _forget_device() -> None:
    global _raw_stream, _device
    _raw_stream = _device = None


os.register_at_fork(after_in_child=_forget_device)       # (torch refuses a device that the parent has initialised)


class Proj:
    """One projection descriptor; keeps the tensors it points to alive."""

    def __init__(self, K: int, N: int, group: int, w_blob, lora_a=None, lora_b=None,
                 alpha: float = 1.0, n_adapters: Optional[int] = None, rank: Optional[int] = None):
        self.K, self.N, self.group = int(K), int(N), int(group)
        self.w_blob, self.lora_a, self.lora_b = w_blob, lora_a, lora_b
        self.alpha = float(alpha)
        if lora_a is not None:
            self.n_adapters = int(lora_a.shape[0]) if n_adapters is None else int(n_adapters)
            self.rank = int(lora_a.shape[1]) if rank is None else int(rank)
        else:
            self.n_adapters = 0 if n_adapters is None else int(n_adapters)
            self.rank = 0 if rank is None else int(rank)

    def struct(self) -> _ProjStruct:
        return _ProjStruct(self.K, self.N, self.group, _ptr(self.w_blob), self.n_adapters,
                           self.rank, _ptr(self.lora_a), _ptr(self.lora_b), self.alpha)


def _proj_array(projs: Sequence[Proj]):
    arr = (_ProjStruct * len(projs))()
    for i, p in enumerate(projs):
        arr[i] = p.struct()
    return arr


def blob_bytes(K: int, N: int, group: int) -> int:
    return int(load_library().mlora_w4_blob_bytes(K, N, group))


def prepack(K: int, N: int, group: int, wq, scales_f16, w_blob) -> None:
    _check(load_library().mlora_w4_prepack(K, N, group, _ptr(wq), _ptr(scales_f16), _ptr(w_blob),
                                           _stream()), "mlora_w4_prepack")


def unpack(proj: Proj, codes=None, w_f32=None) -> None:
    st = proj.struct()
    _check(load_library().mlora_w4_unpack(C.byref(st), _ptr(codes), _ptr(w_f32), _stream()),
           "mlora_w4_unpack")


def group_rows(row_adapter, M: int, n_adapters: int, perm, seg_adapter, seg_start, n_seg) -> None:
    _check(load_library().mlora_group_rows(_ptr(row_adapter), M, n_adapters, _ptr(perm),
                                           _ptr(seg_adapter), _ptr(seg_start), _ptr(n_seg),
                                           _stream()), "mlora_group_rows")


def workspace_init(workspace) -> None:
    n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load_library().mlora_w4_workspace_init(_ptr(workspace), n, _stream()),
           "mlora_w4_workspace_init")


def workspace_status(workspace) -> int:
    """Status word of a workspace (0 = no block gave up waiting); waits for the current stream."""
    word = C.c_int32(-1)
    _check(load_library().mlora_w4_workspace_status(_ptr(workspace), C.byref(word), _stream()),
           "mlora_w4_workspace_status")
    return int(word.value)


def debug_spin_limit(limit: int) -> int:
    return int(load_library().mlora_w4_debug_spin_limit(int(limit)))


def workspace_bytes(projs: Sequence[Proj], M: int) -> int:
    arr = _proj_array(projs)
    return int(load_library().mlora_w4_workspace_bytes(arr, len(projs), M))


def layer_step_plan(projs: Sequence[Proj], M: int) -> dict:
    """How the library would run a call over these projections (see mlora_w4_layer_step_plan)."""
    arr = _proj_array(projs)
    info = (C.c_int32 * 5)()
    _check(load_library().mlora_w4_layer_step_plan(arr, len(projs), M, info), "mlora_w4_layer_step_plan")
    return {"launches": info[0], "wide": bool(info[1]), "rows_per_chunk": info[2],
            "grid_x": info[3], "grid_z": info[4]}


def layer_step_block_rows(projs: Sequence[Proj], M: int, int8_rows: bool = False) -> int:
    """Rows per base block of such a call's first launch (see mlora_w4_layer_step_block_rows)."""
    return load_library().mlora_w4_layer_step_block_rows(_proj_array(projs), len(projs), M, int(int8_rows))


def layer_step_waves_per_tile(projs: Sequence[Proj], M: int, int8_rows: bool = False) -> int:
    """Waves that share a column tile in such a call's first launch (see mlora_w4_layer_step_waves_per_tile)."""
    return load_library().mlora_w4_layer_step_waves_per_tile(_proj_array(projs), len(projs), M, int(int8_rows))


def linear(proj: Proj, x, row_adapter, M: int, y, y_dtype: int = Y_BF16, workspace=None) -> None:
    st = proj.struct()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load_library().mlora_w4_linear(C.byref(st), _ptr(x), _ptr(row_adapter), M, _ptr(y),
                                          y_dtype, _ptr(workspace), ws_bytes, _stream()),
           "mlora_w4_linear")


class LayerPlan:
    """Marshalled arguments of a layer_step call, reusable across calls (no per-call Python
    allocation in timing loops)."""

    def __init__(self, projs: Sequence[Proj], xs: Sequence, ys: Sequence, row_adapter, M: int,
                 y_dtype: int, workspace):
        assert len(projs) == len(xs) == len(ys)
        self.keep = (list(projs), list(xs), list(ys), row_adapter, workspace)
        self.n = len(projs)
        self.arr = _proj_array(projs)
        self.xs = (C.c_void_p * self.n)(*[_ptr(x) for x in xs])
        self.ys = (C.c_void_p * self.n)(*[_ptr(y) for y in ys])
        self.rows = _ptr(row_adapter)
        self.M, self.y_dtype = int(M), int(y_dtype)
        self.ws = _ptr(workspace)
        self.ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self.fn = load_library().mlora_w4_layer_step

    def run(self, stream: Optional[int] = None) -> None:
        st = self.fn(self.arr, self.n, self.xs, self.ys, self.rows, self.M, self.y_dtype,
                     self.ws, self.ws_bytes, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, "mlora_w4_layer_step")


PAIR_NONE, PAIR_ROPE, PAIR_SWIGLU = 0, 1, 2


class Epilogue:
    """What a fused call does to one projection's outputs (mlora_w4_epilogue); keeps its tensors."""

    def __init__(self, row_scale=None, pair_op: int = PAIR_NONE, rope_cos=None, rope_sin=None, residual=None,
                 sq_in=None, sq_parts: int = 0, sq_eps: float = 0.0, sq_out=None):
        self.keep = (row_scale, rope_cos, rope_sin, residual, sq_in, sq_out)
        self.struct = _EpilogueStruct(_ptr(row_scale), pair_op, _ptr(rope_cos), _ptr(rope_sin), _ptr(residual),
                                      _ptr(sq_in), int(sq_parts), float(sq_eps), _ptr(sq_out))


class LayerPlanFused:
    """Marshalled arguments of mlora_w4_layer_step_fused."""

    def __init__(self, projs: Sequence[Proj], epis: Sequence[Epilogue], xs: Sequence, ys: Sequence, row_adapter,
                 M: int, y_dtype: int, workspace):
        assert len(projs) == len(xs) == len(ys) == len(epis)
        self.keep = (list(projs), list(epis), list(xs), list(ys), row_adapter, workspace)
        self.n = len(projs)
        self.arr = _proj_array(projs)
        self.epis = (_EpilogueStruct * self.n)(*[e.struct for e in epis])
        self.xs = (C.c_void_p * self.n)(*[_ptr(x) for x in xs])
        self.ys = (C.c_void_p * self.n)(*[_ptr(y) for y in ys])
        self.rows = _ptr(row_adapter)
        self.M, self.y_dtype = int(M), int(y_dtype)
        self.ws = _ptr(workspace)
        self.ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self.fn = load_library().mlora_w4_layer_step_fused

    def run(self, stream: Optional[int] = None) -> None:
        st = self.fn(self.arr, self.epis, self.n, self.xs, self.ys, self.rows, self.M, self.y_dtype,
                     self.ws, self.ws_bytes, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, "mlora_w4_layer_step_fused")


def rms_scale(x, M: int, K: int, eps: float, scale, stream: Optional[int] = None) -> None:
    _check(load_library().mlora_rms_scale(_ptr(x), M, K, float(eps), _ptr(scale),
                                          _stream() if stream is None else stream), "mlora_rms_scale")


def lora_int16_expand(a_q, b_q, n_adapters: int, rank: int, K: int, N: int, alpha: float, s_a: float, s_b: float,
                      lora_a, lora_b, stream: Optional[int] = None) -> float:
    """int16 LoRA stacks -> the bf16 tensors of a pair of four times the rank (written to lora_a,
    lora_b); returns the alpha to use with them."""
    alpha_out = C.c_float(0.0)
    _check(load_library().mlora_lora_int16_expand(_ptr(a_q), _ptr(b_q), n_adapters, rank, K, N, float(alpha),
                                                  float(s_a), float(s_b), _ptr(lora_a), _ptr(lora_b),
                                                  C.byref(alpha_out), _stream() if stream is None else stream),
           "mlora_lora_int16_expand")
    return float(alpha_out.value)


def a8_workspace_bytes(projs: Sequence[Proj], M: int) -> int:
    arr = _proj_array(projs)
    return int(load_library().mlora_w4a8_workspace_bytes(arr, len(projs), M))


class LayerPlanA8:
    """Marshalled arguments of mlora_w4a8_layer_step (int8 activations, one scale per tensor)."""

    def __init__(self, projs: Sequence[Proj], xs: Sequence, x_scales: Sequence[float], ys: Sequence,
                 row_adapter, M: int, y_dtype: int, workspace):
        assert len(projs) == len(xs) == len(ys) == len(x_scales)
        self.keep = (list(projs), list(xs), list(ys), row_adapter, workspace)
        self.n = len(projs)
        self.arr = _proj_array(projs)
        self.xs = (C.c_void_p * self.n)(*[_ptr(x) for x in xs])
        self.ys = (C.c_void_p * self.n)(*[_ptr(y) for y in ys])
        self.scales = (C.c_float * self.n)(*[float(v) for v in x_scales])
        self.rows = _ptr(row_adapter)
        self.M, self.y_dtype = int(M), int(y_dtype)
        self.ws = _ptr(workspace)
        self.ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        self.fn = load_library().mlora_w4a8_layer_step

    def run(self, stream: Optional[int] = None) -> None:
        st = self.fn(self.arr, self.n, self.xs, self.scales, self.ys, self.rows, self.M, self.y_dtype,
                     self.ws, self.ws_bytes, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, "mlora_w4a8_layer_step")


def layer_step_static(projs: Sequence[Proj], xs: Sequence, ys: Sequence, row_adapter, M: int,
                      y_dtype: int = Y_BF16) -> None:
    """mlora_w4_layer_step_static: the library's built-in scratch instead of a workspace."""
    n = len(projs)
    assert n == len(xs) == len(ys)
    arr = _proj_array(projs)
    cxs = (C.c_void_p * n)(*[_ptr(x) for x in xs])
    cys = (C.c_void_p * n)(*[_ptr(y) for y in ys])
    _check(load_library().mlora_w4_layer_step_static(arr, n, cxs, cys, _ptr(row_adapter), int(M),
                                                     int(y_dtype), _stream()),
           "mlora_w4_layer_step_static")


def layer_step(projs: Sequence[Proj], xs: Sequence, ys: Sequence, row_adapter, M: int,
               y_dtype: int = Y_BF16, workspace=None) -> None:
    LayerPlan(projs, xs, ys, row_adapter, M, y_dtype, workspace).run()


class TreeAttention:
    """Descriptor of a masked tree attention call (include/mlora_tree_attention.h); keeps the
    tensors it points to alive.  Tensors are torch device tensors in the layouts of the header."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, n_streams: int, rows_per_stream: int,
                 scale: float, k_prefill, v_prefill, k_fprefix, v_fprefix, k_stream, v_stream, len_stream,
                 k_new, v_new, parent, is_forecast, len_prefill: int, len_fprefix: int, cap_stream: int):
        self.keep = (k_prefill, v_prefill, k_fprefix, v_fprefix, k_stream, v_stream, len_stream, k_new, v_new,
                     parent, is_forecast)
        self.shape = (n_streams * rows_per_stream, n_q_heads, head_dim)
        self.struct = _TreeAttnStruct(n_q_heads, n_kv_heads, head_dim, n_streams, rows_per_stream, scale,
                                      _ptr(k_prefill), _ptr(v_prefill), len_prefill,
                                      _ptr(k_fprefix), _ptr(v_fprefix), len_fprefix,
                                      _ptr(k_stream), _ptr(v_stream), cap_stream, _ptr(len_stream),
                                      _ptr(k_new), _ptr(v_new), _ptr(parent), _ptr(is_forecast))

    def workspace_bytes(self) -> int:
        return int(load_library().mlora_tree_attention_workspace_bytes(C.byref(self.struct)))

    def plan(self) -> dict:
        """How the library would run the call (see mlora_tree_attention_plan)."""
        info = (C.c_int32 * 3)()
        _check(load_library().mlora_tree_attention_plan(C.byref(self.struct), info), "mlora_tree_attention_plan")
        return {"tiles": info[0], "waves": info[1], "splits": info[2]}

    def run(self, q, out, out_dtype: int, workspace, stream: Optional[int] = None) -> None:
        n = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _check(load_library().mlora_tree_attention(C.byref(self.struct), _ptr(q), _ptr(out), out_dtype,
                                                   _ptr(workspace), n, _stream() if stream is None else stream),
               "mlora_tree_attention")


def ds2d_rows(branch: Sequence[int], n_forecast: int):
    """(tokens, rows) of one stream for a branch configuration (mlora_ds2d_rows)."""
    arr = (C.c_int32 * max(1, len(branch)))(*[int(b) for b in branch])
    t, r = C.c_int32(0), C.c_int32(0)
    _check(load_library().mlora_ds2d_rows(arr, len(branch), n_forecast, C.byref(t), C.byref(r)), "mlora_ds2d_rows")
    return int(t.value), int(r.value)


def ds2d_layout(branch: Sequence[int], n_forecast: int):
    """(parent, is_forecast, level) lists of one stream (mlora_ds2d_layout)."""
    _, rows = ds2d_rows(branch, n_forecast)
    arr = (C.c_int32 * max(1, len(branch)))(*[int(b) for b in branch])
    parent, level = (C.c_int32 * rows)(), (C.c_int32 * rows)()
    is_forecast = (C.c_uint8 * rows)()
    _check(load_library().mlora_ds2d_layout(arr, len(branch), n_forecast, parent, is_forecast, level),
           "mlora_ds2d_layout")
    return list(parent), list(is_forecast), list(level)


class Ds2dStep:
    """Descriptor of mlora_ds2d_step (include/mlora_ds2d.h)."""

    def __init__(self, n_streams: int, n_forecast: int, branch: Sequence[int], next_branch: Sequence[int],
                 vocab: int, logits_dtype: int):
        st = _Ds2dStruct()
        st.n_streams, st.n_forecast, st.depth, st.next_depth = n_streams, n_forecast, len(branch), len(next_branch)
        for i, b in enumerate(branch):
            st.branch[i] = int(b)
        for i, b in enumerate(next_branch):
            st.next_branch[i] = int(b)
        st.vocab, st.logits_dtype = vocab, logits_dtype
        self.struct = st

    def workspace_bytes(self) -> int:
        return int(load_library().mlora_ds2d_workspace_bytes(C.byref(self.struct)))

    def late_drafts(self) -> bool:
        """Whether the step reads the forecast rows after the walk (see mlora_ds2d_late_drafts)."""
        return bool(load_library().mlora_ds2d_late_drafts(C.byref(self.struct)))

    def run(self, logits, tokens, n_accepted, accepted_rows, emitted, next_tokens, workspace,
            stream: Optional[int] = None) -> None:
        n = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _check(load_library().mlora_ds2d_step(C.byref(self.struct), _ptr(logits), _ptr(tokens), _ptr(n_accepted),
                                              _ptr(accepted_rows), _ptr(emitted), _ptr(next_tokens),
                                              _ptr(workspace), n, _stream() if stream is None else stream),
               "mlora_ds2d_step")


ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_TURNS = 0, 1, 2, 3
_EINVAL, _ESHAPE, _EWORKSPACE = -1, -2, -4


class _Kind:
    """Types that a buffer's elements may have, by name; `last` is the one that was met last."""

    def __init__(self, itemsize: int, *names: str):
        self.itemsize, self.names, self.last = itemsize, {"torch." + n for n in names}, None

    def takes(self, dtype) -> bool:
        if dtype is not self.last:
            if str(dtype) not in self.names:
                return False
            self.last = dtype
        return True


_AS_BF16 = _Kind(2, "bfloat16", "int16", "uint16")       # (or their patterns)
_AS_FP32, _AS_FP64 = _Kind(4, "float32"), _Kind(8, "float64")
_AS_INT32 = _Kind(4, "int32", "uint32")
_AS_INT8 = _Kind(1, "int8")


def _buffer(t, where: str, kind: _Kind, shape=None, n: Optional[int] = None) -> None:
    """Refuses what is no dense device tensor of elements of this kind, of this shape or number of elements."""
    if not t.is_cuda or not kind.takes(t.dtype) or not t.is_contiguous():
        raise MloraError(_EINVAL, where)
    if (shape is not None and tuple(t.shape) != tuple(shape)) or (n is not None and t.numel() != n):
        raise MloraError(_ESHAPE, where)


def _call_buffer(t, where: str, kind: _Kind, n: int) -> None:
    """_buffer for what changes from call to call: one look, and the reason only if something is wrong or new."""
    if t.nbytes != kind.itemsize * n or t.dtype is not kind.last or not t.is_contiguous() or not t.is_cuda:
        _buffer(t, where, kind, n=n)


class Rope:
    """Rotary positions (mlora_rope): `rot` of head_dim features turn, in pairs of the half or the interleaved layout, by
    frequencies that are plain, divided by factor (linear), of a larger base (base) or stretched where they turn fewer than
    low..high times within context positions (turns).  Keeps the table of the frequencies, on the device where it is to be used."""

    def __init__(self, head_dim: int, rot: int, layout: int = ROPE_HALF, scaling: int = ROPE_PLAIN, theta: float = 10000.0,
                 factor: float = 1.0, low: float = 1.0, high: float = 4.0, context: float = 8192.0, device="cuda:0"):
        import torch
        self.struct = _RopeStruct(int(head_dim), int(rot), int(layout), int(scaling), float(theta), float(factor),
                                  float(low), float(high), float(context))
        freq = (C.c_double * max(1, int(rot) // 2))()
        _check(load_library().mlora_rope_frequencies(C.byref(self.struct), freq), "mlora_rope_frequencies")
        self.quarter_turns = torch.tensor(list(freq), dtype=torch.float64).to(device)

    def rows(self, M: int, rows_per_stream: Optional[int], base, offset) -> _RopeRowsStruct:
        R = int(M if rows_per_stream is None else rows_per_stream)
        _buffer(self.quarter_turns, "rope frequencies", _AS_FP64)
        if base is not None:
            _buffer(base, "rope base", _AS_INT32, n=M // max(1, R))
        if offset is not None:
            _buffer(offset, "rope offset", _AS_INT32, n=R)
        return _RopeRowsStruct(int(M), max(1, R), _ptr(base), _ptr(offset), _ptr(self.quarter_turns))


class RopeTables:
    """Marshalled arguments of mlora_rope_tables: cos and sin fp32 [M][rot / 2] of rows at base[stream] + offset[row]."""

    def __init__(self, rope: Rope, cos, sin, M: int, rows_per_stream: Optional[int] = None, base=None, offset=None):
        for t in (cos, sin):
            _buffer(t, "mlora_rope_tables", _AS_FP32, n=M * (rope.struct.rot // 2))
        self.keep = (rope, cos, sin, base, offset)
        self.rows = rope.rows(M, rows_per_stream, base, offset)
        self.args = (C.byref(rope.struct), C.byref(self.rows), _ptr(cos), _ptr(sin))
        self.fn = load_library().mlora_rope_tables

    def run(self, stream: Optional[int] = None) -> None:
        st = self.fn(*self.args, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, "mlora_rope_tables")


class RopeTensor:
    """One tensor of a RopePlan: x and y [M][heads][head_dim], any strides with the features next to each other; y may be x.
    Without rotate its rows are copied."""

    def __init__(self, x, y, rotate: bool = True):
        for t in (x, y):
            if not t.is_cuda or t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
                raise MloraError(_EINVAL, "rope tensor")
        if x.shape != y.shape or x.dtype != y.dtype:
            raise MloraError(_ESHAPE, "rope tensor")
        self.x, self.y = x, y
        self.struct = _RopeTensorStruct(_ptr(x), _ptr(y), x.stride(0), x.stride(1), y.stride(0), y.stride(1),
                                        int(x.shape[1]), int(bool(rotate)))


class RopePlan:
    """Marshalled arguments of mlora_rope_apply: all tensors turned (inverse: back) in one launch."""

    def __init__(self, rope: Rope, tensors: Sequence[RopeTensor], M: int, dtype: int, inverse: bool = False,
                 rows_per_stream: Optional[int] = None, base=None, offset=None):
        for t in tensors:
            if t.x.shape[0] != M or t.x.shape[2] != rope.struct.head_dim:
                raise MloraError(_ESHAPE, "mlora_rope_apply")
            if not (_AS_BF16 if dtype == Y_BF16 else _AS_FP32).takes(t.x.dtype):
                raise MloraError(_EINVAL, "mlora_rope_apply")
        self.keep = (rope, list(tensors), base, offset)
        self.rows = rope.rows(M, rows_per_stream, base, offset)
        self.arr = (_RopeTensorStruct * max(1, len(tensors)))(*[t.struct for t in tensors])
        self.args = (C.byref(rope.struct), C.byref(self.rows), self.arr, len(tensors), int(dtype), int(bool(inverse)))
        self.fn = load_library().mlora_rope_apply

    def run(self, stream: Optional[int] = None) -> None:
        st = self.fn(*self.args, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, "mlora_rope_apply")


class StreamCache:
    """The streams' cache segments of all layers (mlora_stream_cache): k and v bf16 [L][S][H][cap][head_dim], mass fp32 and
    slot_pos int32 [L][S][H][cap], len and next_pos int32 [S].  k[l], v[l] and len are what TreeAttention takes as
    k_stream, v_stream and len_stream.  Made outside of a graph capture (its tickets are uploaded here)."""

    def __init__(self, k, v, mass, slot_pos, len, next_pos):
        import torch
        if k.dim() != 5:
            raise MloraError(_ESHAPE, "stream cache")
        L, S, H, cap, D = (int(x) for x in k.shape)
        for t in (k, v):
            _buffer(t, "stream cache", _AS_BF16, (L, S, H, cap, D))
        _buffer(mass, "stream cache", _AS_FP32, (L, S, H, cap))
        _buffer(slot_pos, "stream cache", _AS_INT32, (L, S, H, cap))
        for t in (len, next_pos):
            _buffer(t, "stream cache", _AS_INT32, (S,))
        self.k, self.v, self.mass, self.slot_pos, self.len, self.next_pos = k, v, mass, slot_pos, len, next_pos
        self.tickets = torch.zeros((S, 32), dtype=torch.int32).to(k.device)  # (an upload: done when it returns)
        self.shape = (L, S, H, cap, D)
        self.struct = _StreamCacheStruct(L, S, H, D, cap, _ptr(k), _ptr(v), _ptr(mass), _ptr(slot_pos), _ptr(len),
                                         _ptr(next_pos), _ptr(self.tickets))
        self.ref = C.byref(self.struct)
        self.streams, self.heads, self.row_bytes, self.list_bytes = S, L * S * H, 2 * L * S * H * D, 4 * S
        self.append_fn = load_library().mlora_stream_cache_append
        self.compress_fn = load_library().mlora_stream_cache_compress

    def append(self, k_new, v_new, rows_per_stream: int, rows, budget: int, sink: int = 0, recent: int = 0,
               stream: Optional[int] = None) -> None:
        """Listed rows (int32 [S][n], None: all) of k_new and v_new bf16 [L][S * rows_per_stream][H][head_dim] enter the
        caches; beyond the budget they take the slots of the lowest rank."""
        where = "mlora_stream_cache_append"
        size = self.row_bytes * rows_per_stream
        if (k_new.nbytes != size or v_new.nbytes != size or k_new.dtype is not _AS_BF16.last
                or v_new.dtype is not _AS_BF16.last or not k_new.is_contiguous() or not v_new.is_contiguous()
                or not k_new.is_cuda or not v_new.is_cuda):
            for t in (k_new, v_new):
                _call_buffer(t, where, _AS_BF16, size // 2)
        listed = 0
        if rows is not None:
            size = rows.nbytes
            listed = size // self.list_bytes
            if (size != listed * self.list_bytes or rows.dtype is not _AS_INT32.last or not rows.is_contiguous()
                    or not rows.is_cuda):
                _buffer(rows, where, _AS_INT32, n=self.streams * listed)
            if listed == 0:                              # (its pointer is null: all rows)
                raise MloraError(_ESHAPE, where)
        st = self.append_fn(self.ref, k_new.data_ptr(), v_new.data_ptr(), rows_per_stream,
                            None if rows is None else rows.data_ptr(), listed, budget, sink, recent,
                            _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)

    def compress(self, to: "StreamCache", kept, budget: int, sink: int = 0, recent: int = 0,
                 stream: Optional[int] = None) -> None:
        """The slots of the highest rank, at most budget, to the front of another cache; kept int32 [L][S][H][budget]
        tells which (-1 beyond)."""
        _call_buffer(kept, "mlora_stream_cache_compress", _AS_INT32, self.heads * budget)
        st = self.compress_fn(self.ref, to.ref, kept.data_ptr(), budget, sink, recent,
                              _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, "mlora_stream_cache_compress")


class AttentionMass:
    """Descriptor of mlora_attention_mass_add: attention weights of the newest rows added to the mass of the cache's slots
    and of a prefill segment (k_prefill bf16 [L][H][P][head_dim], mass_prefill fp32 [L][H][P])."""

    def __init__(self, cache: StreamCache, n_q_heads: int, rows_per_stream: int, scale: float, k_prefill=None,
                 mass_prefill=None, decay: float = 1.0):
        L, S, H, _, D = cache.shape
        P = 0
        if k_prefill is not None:
            P = int(k_prefill.shape[2]) if k_prefill.dim() == 4 else -1
            _buffer(k_prefill, "attention mass", _AS_BF16, (L, H, P, D))
            if P > 0 and mass_prefill is None:
                raise MloraError(_EINVAL, "attention mass")
            if mass_prefill is not None:
                _buffer(mass_prefill, "attention mass", _AS_FP32, (L, H, P))
        self.keep = (cache, k_prefill, mass_prefill)
        self.streams, self.list_bytes, self.q_elements = S, 4 * S, L * S * int(rows_per_stream) * int(n_q_heads) * D
        self.struct = _AttentionMassStruct(cache.struct, int(n_q_heads), int(rows_per_stream), float(scale),
                                           _ptr(k_prefill), _ptr(mass_prefill), P, float(decay))
        self.ref = C.byref(self.struct)
        self.fn = load_library().mlora_attention_mass_add

    def workspace_bytes(self, n_rows: int = 0) -> int:
        """For calls with n_rows listed rows per stream, 0: with all rows."""
        return int(load_library().mlora_attention_mass_workspace_bytes(self.ref, n_rows))

    def run(self, q, rows, workspace, stream: Optional[int] = None) -> None:
        """q bf16 [L][S * rows_per_stream][n_q_heads][head_dim], rows int32 [S][n] or None (all)."""
        where = "mlora_attention_mass_add"
        _call_buffer(q, where, _AS_BF16, self.q_elements)
        listed = 0
        if rows is not None:
            size = rows.nbytes
            listed = size // self.list_bytes
            if (size != listed * self.list_bytes or rows.dtype is not _AS_INT32.last or not rows.is_contiguous()
                    or not rows.is_cuda):
                _buffer(rows, where, _AS_INT32, n=self.streams * listed)
            if listed == 0:                              # (its pointer is null: all rows)
                raise MloraError(_ESHAPE, where)
        if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
            raise MloraError(_EINVAL, where)
        st = self.fn(self.ref, q.data_ptr(), None if rows is None else rows.data_ptr(), listed,
                     None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes,
                     _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)


class LogitRules:
    """Descriptor of mlora_logit_rules_apply: penalties for tokens that counts (int32 [S][V]) and the rows' paths hold,
    biases (fp32 [n][V], a row per stream) and grammar masks (bits, int32 [n][(V + 31) / 32], a row per logits row)."""

    def __init__(self, n_streams: int, rows_per_stream: int, tokens_per_stream: int, vocab: int, logits_dtype: int, parent,
                 counts=None, repetition=None, frequency=None, presence=None, bias=None, bias_row=None, masks=None,
                 mask_row=None):
        S, R, T, V = int(n_streams), int(rows_per_stream), int(tokens_per_stream), int(vocab)
        where = "logit rules"
        _buffer(parent, where, _AS_INT32, n=S * R)
        if counts is not None:
            _buffer(counts, where, _AS_INT32, (S, V))
        for t in (repetition, frequency, presence):
            if t is not None:
                _buffer(t, where, _AS_FP32, n=S)
        if (bias is None) != (bias_row is None) or (masks is None) != (mask_row is None):
            raise MloraError(_EINVAL, where)
        if bias is not None:
            _buffer(bias, where, _AS_FP32, (bias.shape[0], V))
            _buffer(bias_row, where, _AS_INT32, n=S)
        if masks is not None:
            _buffer(masks, where, _AS_INT32, (masks.shape[0], (V + 31) // 32))
            _buffer(mask_row, where, _AS_INT32, n=S * R)
        self.keep = (parent, counts, repetition, frequency, presence, bias, bias_row, masks, mask_row)
        self.streams, self.tokens, self.logits, self.kind = S, S * T, S * R * V, _AS_BF16 if logits_dtype == Y_BF16 else _AS_FP32
        self.list_bytes, self.token_bytes, self.logit_bytes = 4 * S, 4 * self.tokens, self.kind.itemsize * self.logits
        self.struct = _LogitRulesStruct(S, R, T, V, int(logits_dtype), _ptr(parent), _ptr(counts), _ptr(repetition),
                                        _ptr(frequency), _ptr(presence), _ptr(bias), _ptr(bias_row),
                                        0 if bias is None else int(bias.shape[0]), _ptr(masks), _ptr(mask_row),
                                        0 if masks is None else int(masks.shape[0]))
        self.ref = C.byref(self.struct)
        self.fn = load_library().mlora_logit_rules_apply

    def run(self, logits, tokens, out, new_tokens=None, stream: Optional[int] = None) -> None:
        """logits [S * R][V] -> out (may be logits itself); tokens int32 [S][T]; new_tokens int32 [S][n]: counted first."""
        where = "mlora_logit_rules_apply"
        kind, size = self.kind, self.logit_bytes
        dtype = kind.last
        if (logits.nbytes != size or out.nbytes != size or tokens.nbytes != self.token_bytes or logits.dtype is not dtype
                or out.dtype is not dtype or tokens.dtype is not _AS_INT32.last or not logits.is_contiguous()
                or not out.is_contiguous() or not tokens.is_contiguous() or not logits.is_cuda or not out.is_cuda
                or not tokens.is_cuda):
            _call_buffer(logits, where, kind, self.logits)
            _call_buffer(out, where, kind, self.logits)
            _call_buffer(tokens, where, _AS_INT32, self.tokens)
        fresh = 0
        if new_tokens is not None:
            size = new_tokens.nbytes
            fresh = size // self.list_bytes
            if (size != fresh * self.list_bytes or new_tokens.dtype is not _AS_INT32.last or not new_tokens.is_contiguous()
                    or not new_tokens.is_cuda):
                _buffer(new_tokens, where, _AS_INT32, n=self.streams * fresh)
        st = self.fn(self.ref, logits.data_ptr(), tokens.data_ptr(), new_tokens.data_ptr() if fresh else None, fresh,
                     out.data_ptr(), _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)


PAGE_TOKENS = 64


class PageCache:
    """A paged cache of 8 bits (mlora_page_cache): k int8 [L][n_pages][H][64][head_dim], v int8 [L][n_pages][H][head_dim][64], scales fp32
    [L][n_pages][H], tails bf16 [L][S][H][64][head_dim], slot and len int32 [S], table int32 [S][max_pages], refs int32
    [n_pages].  Made outside of a graph capture (the library's own words are uploaded here).  A program that writes refs itself, as in going back to a
    state that it kept, calls refs_written() before the next append."""

    def __init__(self, k, v, k_scale, v_scale, k_tail, v_tail, slot, len, table, refs):
        import torch
        where = "page cache"
        if k.dim() != 5 or k_tail.dim() != 5 or table.dim() != 2:
            raise MloraError(_ESHAPE, where)
        L, N, H, tokens, D = (int(x) for x in k.shape)
        S, columns = int(k_tail.shape[1]), int(table.shape[1])
        if tokens != PAGE_TOKENS:
            raise MloraError(_ESHAPE, where)
        _buffer(k, where, _AS_INT8, (L, N, H, tokens, D))
        _buffer(v, where, _AS_INT8, (L, N, H, D, tokens))
        for t in (k_scale, v_scale):
            _buffer(t, where, _AS_FP32, (L, N, H))
        for t in (k_tail, v_tail):
            _buffer(t, where, _AS_BF16, (L, S, H, tokens, D))
        for t, shape in ((slot, (S,)), (len, (S,)), (table, (S, columns)), (refs, (N,))):
            _buffer(t, where, _AS_INT32, shape)
        words = int(load_library().mlora_page_cache_own_words(S, N))
        if words == 0:
            raise MloraError(_ESHAPE, where)
        self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail = k, v, k_scale, v_scale, k_tail, v_tail
        self.slot, self.len, self.table, self.refs = slot, len, table, refs
        self.own = torch.zeros(words, dtype=torch.int32).to(k.device)       # (an upload: done when it returns)
        self.shape = (L, S, H, D)
        self.struct = _PageCacheStruct(L, S, H, D, N, columns, _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(k_tail),
                                       _ptr(v_tail), _ptr(slot), _ptr(len), _ptr(table), _ptr(refs), _ptr(self.own))
        self.ref = C.byref(self.struct)
        self.streams, self.row_bytes, self.list_bytes = S, 2 * L * S * H * D, 4 * S
        lib = load_library()
        self.append_fn, self.reorder_fn, self.copy_fn = lib.mlora_page_cache_append, lib.mlora_page_cache_reorder, lib.mlora_page_cache_copy

    @classmethod
    def empty(cls, n_layers: int, n_streams: int, n_kv_heads: int, head_dim: int, n_pages: int, max_pages: int, device="cuda:0") -> "PageCache":
        """An empty cache, its memory made here."""
        import torch
        L, S, H, D, N, P = n_layers, n_streams, n_kv_heads, head_dim, n_pages, PAGE_TOKENS
        z = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=device)   # noqa: E731
        return cls(z((L, N, H, P, D), torch.int8), z((L, N, H, D, P), torch.int8), z((L, N, H), torch.float32), z((L, N, H), torch.float32),
                   z((L, S, H, P, D), torch.bfloat16), z((L, S, H, P, D), torch.bfloat16), torch.arange(S, dtype=torch.int32).to(device),
                   z((S,), torch.int32), torch.full((S, max_pages), -1, dtype=torch.int32).to(device), z((N,), torch.int32))

    def refs_written(self) -> None:
        """refs was written from outside: the search for free pages starts from the pool's first again (otherwise pages that became free below where it
        had come to are not found).  On the current stream, in a graph as well."""
        self.own[:1].zero_()

    def append(self, k_new, v_new, rows_per_stream: int, rows=None, appended=None, stream: Optional[int] = None) -> None:
        """Listed rows (int32 [S][n], None: all) of k_new and v_new bf16 [L][S * rows_per_stream][H][head_dim] enter; appended
        int32 [S]: how many did."""
        where = "mlora_page_cache_append"
        size = self.row_bytes * rows_per_stream
        if (k_new.nbytes != size or v_new.nbytes != size or k_new.dtype is not _AS_BF16.last
                or v_new.dtype is not _AS_BF16.last or not k_new.is_contiguous() or not v_new.is_contiguous()
                or not k_new.is_cuda or not v_new.is_cuda):
            for t in (k_new, v_new):
                _call_buffer(t, where, _AS_BF16, size // 2)
        listed = 0
        if rows is not None:
            size = rows.nbytes
            listed = size // self.list_bytes
            if (size != listed * self.list_bytes or rows.dtype is not _AS_INT32.last or not rows.is_contiguous()
                    or not rows.is_cuda):
                _buffer(rows, where, _AS_INT32, n=self.streams * listed)
            if listed == 0:                              # (its pointer is null: all rows)
                raise MloraError(_ESHAPE, where)
        if appended is not None:
            _call_buffer(appended, where, _AS_INT32, self.streams)
        st = self.append_fn(self.ref, k_new.data_ptr(), v_new.data_ptr(), rows_per_stream,
                            None if rows is None else rows.data_ptr(), listed, None if appended is None else appended.data_ptr(),
                            _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)

    def reorder(self, source=None, window: int = 0, sink: int = 0, stream: Optional[int] = None) -> None:
        """Stream s becomes what source[s] was (int32 [S]; outside: empty; None: all stay); window > 0: pages that it has left
        behind, but for those of the first `sink` tokens, are given up."""
        where = "mlora_page_cache_reorder"
        if source is not None:
            _call_buffer(source, where, _AS_INT32, self.streams)
        st = self.reorder_fn(self.ref, None if source is None else source.data_ptr(), window, sink,
                             _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)

    def copy_from(self, other: "PageCache", source, n_used=None, stream: Optional[int] = None) -> None:
        """Stream i becomes what source[i] of another cache is (int32 [S]); all that this one held is gone.  n_used int32 [1]:
        pages that the streams hold."""
        where = "mlora_page_cache_copy"
        _call_buffer(source, where, _AS_INT32, self.streams)
        if n_used is not None:
            _call_buffer(n_used, where, _AS_INT32, 1)
        st = self.copy_fn(other.ref, self.ref, source.data_ptr(), None if n_used is None else n_used.data_ptr(),
                          _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)


class PageAttention:
    """Descriptor of mlora_page_attention for one layer of a PageCache: k_new and v_new bf16 [S * R][H][head_dim], parent int32
    [S * R]; takes the place of a TreeAttention in a DecoderLayerStep."""

    def __init__(self, cache: PageCache, layer: int, n_q_heads: int, rows_per_stream: int, scale: float, k_new, v_new, parent,
                 window: int = 0, sink: int = 0):
        L, S, H, D = cache.shape
        M, where = S * int(rows_per_stream), "page attention"
        for t in (k_new, v_new):
            _buffer(t, where, _AS_BF16, n=M * H * D)
        _buffer(parent, where, _AS_INT32, n=M)
        self.keep = (cache, None, None, None, None, None, None, k_new, v_new, parent)
        self.shape = (M, int(n_q_heads), D)
        self.elements = M * int(n_q_heads) * D
        self.struct = _PageAttnStruct(cache.struct, int(layer), int(n_q_heads), int(rows_per_stream), float(scale), int(window), int(sink),
                                      _ptr(k_new), _ptr(v_new), _ptr(parent))
        self.ref = C.byref(self.struct)
        self.fn = load_library().mlora_page_attention

    def workspace_bytes(self) -> int:
        return int(load_library().mlora_page_attention_workspace_bytes(self.ref))

    def plan(self) -> dict:
        """How the library would run the call (see mlora_page_attention_plan)."""
        info = (C.c_int32 * 3)()
        _check(load_library().mlora_page_attention_plan(self.ref, info), "mlora_page_attention_plan")
        return {"tiles": info[0], "waves": info[1], "splits": info[2]}

    def run(self, q, out, out_dtype: int, workspace, stream: Optional[int] = None) -> None:
        """q bf16 [S * R][n_q_heads][head_dim] -> out, the same shape."""
        where = "mlora_page_attention"
        _call_buffer(q, where, _AS_BF16, self.elements)
        _call_buffer(out, where, _AS_FP32 if out_dtype == Y_FP32 else _AS_BF16, self.elements)
        if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
            raise MloraError(_EINVAL, where)
        st = self.fn(self.ref, q.data_ptr(), out.data_ptr(), out_dtype, None if workspace is None else workspace.data_ptr(),
                     0 if workspace is None else workspace.nbytes, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)


class BeamSelect:
    """Descriptor of mlora_beam_select: the best n_beams continuations of every group of n_beams beams."""

    def __init__(self, n_groups: int, n_beams: int, vocab: int, logits_dtype: int, eos: int = -1, pad: int = 0, length_power: float = 0.0):
        self.rows = int(n_groups) * int(n_beams)
        self.kind = _AS_BF16 if logits_dtype == Y_BF16 else _AS_FP32
        self.logits, self.row_bytes = self.rows * int(vocab), 4 * self.rows
        self.struct = _BeamStruct(int(n_groups), int(n_beams), int(vocab), int(logits_dtype), int(eos), int(pad), float(length_power))
        self.ref = C.byref(self.struct)
        self.fn = load_library().mlora_beam_select

    def workspace_bytes(self) -> int:
        return int(load_library().mlora_beam_workspace_bytes(self.ref))

    def run(self, logits, score, length, finished, source, token, score_out, length_out, finished_out, workspace,
            stream: Optional[int] = None) -> None:
        """logits [rows][vocab]; score fp32, length and finished int32 [rows] -> source and token int32 [rows], and the new beams'
        score, length and finished, which may be the old ones' tensors."""
        where = "mlora_beam_select"
        _call_buffer(logits, where, self.kind, self.logits)
        for t in (score, score_out):
            _call_buffer(t, where, _AS_FP32, self.rows)
        for t in (length, finished, source, token, length_out, finished_out):
            _call_buffer(t, where, _AS_INT32, self.rows)
        if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
            raise MloraError(_EINVAL, where)
        st = self.fn(self.ref, logits.data_ptr(), score.data_ptr(), length.data_ptr(), finished.data_ptr(), source.data_ptr(), token.data_ptr(),
                     score_out.data_ptr(), length_out.data_ptr(), finished_out.data_ptr(), None if workspace is None else workspace.data_ptr(),
                     0 if workspace is None else workspace.nbytes, _stream() if stream is None else stream)
        if st != 0:
            raise MloraError(st, where)
