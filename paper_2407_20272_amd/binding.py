"""ctypes binding of libee_decode.so: the same entry points as include/ee_decode.h, argument marshalling only.

Every step of the decode path runs in the library's HIP kernels; torch is used here for device memory and for
the current HIP stream.  There is no CPU fallback: if the library is missing or no GPU is present the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libee_decode.so")

EE_OK = 0
EE_ERR_INVALID_ARG, EE_ERR_SHAPE, EE_ERR_UNSUPPORTED, EE_ERR_WORKSPACE, EE_ERR_HIP = -1, -2, -3, -4, -5
EE_FP32, EE_BF16 = 0, 1
EE_PACK_PLAIN, EE_PACK_QKV, EE_PACK_GATE_UP = 0, 1, 2
EXPORTS = ["ee_last_error", "ee_packed_weight_bytes", "ee_pack_weight", "ee_workspace_bytes", "ee_decode_iteration",
           "ee_exit_check", "ee_kv_fill", "ee_paged_attention_decode", "ee_profile_enable", "ee_profile_read", "ee_calibration_copy",
           "ee_noalloc_init", "ee_exit_check_noalloc_bytes", "ee_exit_check_noalloc", "ee_calibration_read", "ee_calibration_mfma",
           "ee_calibration_mfma_tile", "ee_calibration_intake", "ee_rotary_frequencies", "ee_rotary", "ee_kv_quant_append",
           "ee_kv_quant_read", "ee_paged_attention_quant_bytes", "ee_paged_attention_quant", "ee_kv_quant_evict_bytes",
           "ee_kv_quant_evict", "ee_kv_pages_bytes", "ee_kv_pages_fork", "ee_kv_pages_release", "ee_kv_pages_grow", "ee_kv_pages_compact",
           "ee_kv_pages_shared", "ee_kv_copy", "ee_kv_quant_copy", "ee_beam_select_bytes", "ee_beam_select", "ee_reorder_rows",
           "ee_paged_attention_shared_bytes", "ee_paged_attention_shared"]
EE_ROTARY_HALF, EE_ROTARY_INTERLEAVED = 0, 1
EE_ROTARY_PLAIN, EE_ROTARY_LINEAR, EE_ROTARY_TURNS = 0, 1, 2
EE_QUANT_INT8, EE_QUANT_E4M3 = 0, 1
EE_NOALLOC_SCRATCH_BYTES = 8 << 20
KERNEL_CLASSES = ["norm", "qkv", "attention", "o_proj", "gate_up", "down", "head", "combine", "kv_fill", "other"]


class ee_model_desc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("rms_eps", C.c_float),
                ("rope_theta", C.c_float), ("exit_every", C.c_int32), ("logit_scale", C.c_float),
                ("conf_mode", C.c_int32)]


class ee_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("g_attn", "w_qkv", "w_o", "g_ffn", "w_gate_up", "w_down")]


class ee_model(C.Structure):
    _fields_ = [("desc", ee_model_desc), ("embed", C.c_void_p), ("g_final", C.c_void_p), ("w_lm", C.c_void_p),
                ("layers", C.POINTER(ee_layer_weights)), ("w_cls", C.c_void_p), ("b_cls", C.c_void_p)]


class ee_kv_cache(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("num_blocks", C.c_int32), ("block_size", C.c_int32)]


class ee_batch(C.Structure):
    _fields_ = [("batch", C.c_int32), ("tokens", C.c_void_p), ("context_lens", C.c_void_p),
                ("block_tables", C.c_void_p), ("max_blocks", C.c_int32), ("max_context", C.c_int32),
                ("row_table", C.c_void_p)]


class ee_rotary_desc(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("original_context", C.c_int32), ("theta", C.c_double), ("factor", C.c_double), ("turns_low", C.c_double),
                ("turns_high", C.c_double), ("amplitude", C.c_double)]


class ee_rotary_rows(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("in_stride", C.c_int64), ("out_stride", C.c_int64),
                ("n_heads", C.c_int32)]


class ee_quant_cache(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("scales", C.c_void_p), ("n_layers", C.c_int32),
                ("num_blocks", C.c_int32), ("block_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("format", C.c_int32)]


class ee_page_tables(C.Structure):
    _fields_ = [("block_tables", C.c_void_p), ("lens", C.c_void_p), ("rows", C.c_int32), ("max_blocks", C.c_int32)]


class ee_prefix_groups(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("first_row", C.c_void_p), ("shared_blocks", C.c_void_p), ("max_shared", C.c_int32)]


class EEError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ee_decode error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """Loads the native library (once).  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2407_20272_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.ee_last_error.restype = C.c_char_p
        L.ee_packed_weight_bytes.restype = C.c_size_t
        L.ee_packed_weight_bytes.argtypes = [C.c_int32, C.c_int32]
        L.ee_pack_weight.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.ee_workspace_bytes.restype = C.c_size_t
        L.ee_workspace_bytes.argtypes = [C.POINTER(ee_model_desc), C.c_int32, C.c_int32]
        L.ee_decode_iteration.argtypes = [C.POINTER(ee_model), C.POINTER(ee_kv_cache), C.POINTER(ee_batch),
                                          C.POINTER(C.c_float), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ee_exit_check.argtypes = [C.POINTER(ee_model), C.c_int32, C.c_void_p, C.c_int32, C.c_float, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]
        L.ee_exit_check_noalloc.argtypes = L.ee_exit_check.argtypes[:13] + [C.c_void_p]
        L.ee_exit_check_noalloc_bytes.restype = C.c_size_t
        L.ee_exit_check_noalloc_bytes.argtypes = [C.POINTER(ee_model_desc), C.c_int32]
        L.ee_noalloc_init.argtypes = []
        L.ee_kv_fill.argtypes = [C.POINTER(ee_model), C.POINTER(ee_kv_cache), C.POINTER(ee_batch), C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ee_paged_attention_decode.argtypes = [C.POINTER(ee_model_desc), C.POINTER(ee_kv_cache), C.c_int32, C.c_void_p,
                                                C.POINTER(ee_batch), C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ee_calibration_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ee_calibration_copy.restype = C.c_int
        L.ee_calibration_read.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_int32, C.c_void_p]
        L.ee_calibration_read.restype = C.c_int
        L.ee_calibration_mfma.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.ee_calibration_mfma.restype = C.c_int
        L.ee_calibration_mfma_tile.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.ee_calibration_mfma_tile.restype = C.c_int
        L.ee_calibration_intake.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_int32, C.c_int32, C.c_int32,
                                            C.c_void_p, C.c_void_p]
        L.ee_calibration_intake.restype = C.c_int
        L.ee_profile_enable.argtypes = [C.c_int32]
        L.ee_profile_read.argtypes = [C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_float), C.c_int32]
        L.ee_profile_enable.restype = C.c_int
        L.ee_profile_read.restype = C.c_int
        L.ee_rotary_frequencies.argtypes = [C.POINTER(ee_rotary_desc), C.c_void_p, C.c_void_p]
        L.ee_rotary.argtypes = [C.POINTER(ee_rotary_desc), C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(ee_rotary_rows),
                                C.POINTER(ee_rotary_rows), C.c_int32, C.c_void_p]
        L.ee_kv_quant_append.argtypes = [C.POINTER(ee_quant_cache), C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                         C.c_int32, C.POINTER(ee_batch), C.c_void_p]
        L.ee_kv_quant_read.argtypes = [C.POINTER(ee_quant_cache), C.c_int32, C.POINTER(ee_batch), C.c_void_p, C.c_void_p,
                                       C.c_int32, C.c_void_p]
        L.ee_paged_attention_quant_bytes.argtypes = [C.POINTER(ee_quant_cache), C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        L.ee_paged_attention_quant_bytes.restype = C.c_size_t
        L.ee_paged_attention_quant.argtypes = [C.POINTER(ee_quant_cache), C.c_int32, C.c_int32, C.c_void_p, C.POINTER(ee_batch),
                                               C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ee_kv_quant_evict_bytes.argtypes = [C.POINTER(ee_quant_cache), C.c_int32, C.c_int32]
        L.ee_kv_quant_evict_bytes.restype = C.c_size_t
        L.ee_kv_quant_evict.argtypes = [C.POINTER(ee_quant_cache), C.c_int32, C.POINTER(ee_batch), C.c_void_p, C.c_int32, C.c_void_p,
                                        C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_size_t, C.c_void_p]
        pool, tables, i32, ptr, size = [C.c_void_p, C.c_int32], C.POINTER(ee_page_tables), C.c_int32, C.c_void_p, C.c_size_t
        L.ee_kv_pages_bytes.argtypes, L.ee_kv_pages_bytes.restype = [i32, i32], size
        L.ee_kv_pages_fork.argtypes = pool + [tables, ptr, tables, i32, ptr]
        L.ee_kv_pages_release.argtypes = pool + [tables, ptr]
        L.ee_kv_pages_grow.argtypes = pool + [tables, ptr, ptr, ptr, ptr, size, ptr]
        L.ee_kv_pages_compact.argtypes = pool + [tables, ptr, ptr, ptr, ptr, size, ptr]
        L.ee_kv_pages_shared.argtypes = [tables, ptr, i32, ptr, ptr]
        L.ee_kv_copy.argtypes = [C.POINTER(ee_model_desc), C.POINTER(ee_kv_cache), ptr, i32, ptr, ptr]
        L.ee_kv_quant_copy.argtypes = [C.POINTER(ee_quant_cache), ptr, i32, ptr, ptr]
        L.ee_beam_select_bytes.argtypes, L.ee_beam_select_bytes.restype = [i32] * 4, size
        L.ee_beam_select.argtypes = [ptr, C.c_int64, i32, ptr, ptr] + [i32] * 5 + [ptr] * 5 + [size, ptr]
        L.ee_reorder_rows.argtypes = [ptr, C.c_int64, i32, ptr, i32, C.c_int64, ptr, C.c_int64, ptr]
        L.ee_paged_attention_shared_bytes.argtypes, L.ee_paged_attention_shared_bytes.restype = [C.POINTER(ee_model_desc)] + [i32] * 4, size
        L.ee_paged_attention_shared.argtypes = [C.POINTER(ee_model_desc), C.POINTER(ee_kv_cache), i32, i32, ptr, C.POINTER(ee_batch),
                                                C.POINTER(ee_prefix_groups), ptr, ptr, size, ptr]
        for name in ("ee_kv_pages_fork", "ee_kv_pages_release", "ee_kv_pages_grow", "ee_kv_pages_compact", "ee_kv_pages_shared", "ee_kv_copy",
                     "ee_kv_quant_copy", "ee_beam_select", "ee_reorder_rows", "ee_paged_attention_shared"):
            getattr(L, name).restype = C.c_int
        for name in ("ee_rotary_frequencies", "ee_rotary", "ee_kv_quant_append", "ee_kv_quant_read", "ee_paged_attention_quant",
                     "ee_kv_quant_evict"):
            getattr(L, name).restype = C.c_int
        for name in ("ee_pack_weight", "ee_decode_iteration", "ee_exit_check", "ee_kv_fill", "ee_paged_attention_decode",
                     "ee_exit_check_noalloc", "ee_noalloc_init"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(rc: int):
    if rc != EE_OK:
        raise EEError(rc, lib().ee_last_error().decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device pointer arguments must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _i32(t: torch.Tensor) -> torch.Tensor:
    assert t.dtype == torch.int32
    return t


# ------------------------------------------------------------------------------------------------------
# plain wrappers (same names as the C entry points)
# ------------------------------------------------------------------------------------------------------
def make_desc(cfg) -> ee_model_desc:
    return ee_model_desc(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.head_dim, cfg.d_ffn, cfg.vocab,
                         EE_FP32 if cfg.dtype == "fp32" else EE_BF16, cfg.rms_eps, cfg.rope_theta, cfg.exit_every,
                         cfg.logit_scale, cfg.conf_mode)


def ee_last_error() -> str:
    return lib().ee_last_error().decode()


def ee_packed_weight_bytes(n_out: int, n_in: int) -> int:
    return lib().ee_packed_weight_bytes(n_out, n_in)


def ee_pack_weight(w: torch.Tensor, order: int, pair_stride: int = 0) -> torch.Tensor:
    """Returns the MFMA tile-order image of a plain bf16 [n_out][n_in] matrix (a new device tensor)."""
    assert w.dtype == torch.bfloat16 and w.dim() == 2
    n_out, n_in = w.shape
    out = torch.empty(ee_packed_weight_bytes(n_out, n_in) // 2, dtype=torch.bfloat16, device=w.device)
    _check(lib().ee_pack_weight(_ptr(w.contiguous()), n_out, n_in, order, pair_stride, _ptr(out), _stream()))
    return out


def ee_workspace_bytes(desc: ee_model_desc, max_batch: int, max_context: int) -> int:
    return lib().ee_workspace_bytes(C.byref(desc), max_batch, max_context)


class DeviceModel:
    """Device-resident weights in the layouts the library takes, plus the host-side ee_model record."""

    def __init__(self, cfg, weights: Dict, device="cuda"):
        self.cfg = cfg
        self.desc = make_desc(cfg)
        bf = cfg.dtype == "bf16"
        self._keep: List[torch.Tensor] = []

        def dev(t):
            t = t.to(device).contiguous()
            self._keep.append(t)
            return t

        def mat(t, order=EE_PACK_PLAIN, stride=0):
            t = t.to(device).contiguous()
            if bf:
                t = ee_pack_weight(t, order, stride)
            self._keep.append(t)
            return t

        self.embed = dev(weights["embed"])
        self.g_final = dev(weights["g_final"])
        self.w_lm = mat(weights["w_lm"])
        self.layers = (ee_layer_weights * cfg.n_layers)()
        for i, lw in enumerate(weights["layers"]):
            qkv = torch.cat([lw["w_q"].to(device), lw["w_k"].to(device), lw["w_v"].to(device)], 0)
            gu = torch.cat([lw["w_gate"].to(device), lw["w_up"].to(device)], 0)
            L = self.layers[i]
            L.g_attn = dev(lw["g_attn"]).data_ptr()
            L.w_qkv = mat(qkv, EE_PACK_QKV, cfg.head_dim // 2).data_ptr()
            L.w_o = mat(lw["w_o"]).data_ptr()
            L.g_ffn = dev(lw["g_ffn"]).data_ptr()
            L.w_gate_up = mat(gu, EE_PACK_GATE_UP, cfg.d_ffn).data_ptr()
            L.w_down = mat(lw["w_down"]).data_ptr()
            del qkv, gu
        # dedicated-classifier rows and biases (float32 in every dtype), if the weight set has them
        self.w_cls = dev(weights["w_cls"].float()) if "w_cls" in weights else None
        self.b_cls = dev(weights["b_cls"].float()) if "b_cls" in weights else None
        self.c = ee_model(self.desc, self.embed.data_ptr(), self.g_final.data_ptr(), self.w_lm.data_ptr(), self.layers,
                          self.w_cls.data_ptr() if self.w_cls is not None else None,
                          self.b_cls.data_ptr() if self.b_cls is not None else None)
        torch.cuda.synchronize()

    def with_conf_mode(self, conf_mode: int) -> "DeviceModel":
        """The same device weights under another confidence measure (a second host-side record, nothing copied)."""
        import copy
        v = copy.copy(self)
        v.cfg = self.cfg.with_(conf_mode=conf_mode)
        v.desc = make_desc(v.cfg)
        v.c = ee_model(v.desc, self.c.embed, self.c.g_final, self.c.w_lm, self.layers, self.c.w_cls, self.c.b_cls)
        return v


class PagedKV:
    """Paged K/V pools [n_layers][num_blocks][H][16][dh] in the model dtype."""

    def __init__(self, cfg, num_blocks: int, device="cuda", fill: float = 0.0):
        self.cfg, self.num_blocks = cfg, num_blocks
        shape = (cfg.n_layers, num_blocks, cfg.n_heads, cfg.block_size, cfg.head_dim)
        self.k = torch.full(shape, fill, dtype=cfg.torch_dtype, device=device)
        self.v = torch.full(shape, fill, dtype=cfg.torch_dtype, device=device)
        self.c = ee_kv_cache(self.k.data_ptr(), self.v.data_ptr(), num_blocks, cfg.block_size)

    @classmethod
    def of(cls, cfg, k: torch.Tensor, v: torch.Tensor) -> "PagedKV":
        """The record of pools that are there already."""
        c = cls.__new__(cls)
        c.cfg, c.num_blocks, c.k, c.v = cfg, k.shape[1], k, v
        assert k.shape == (cfg.n_layers, c.num_blocks, cfg.n_heads, cfg.block_size, cfg.head_dim) and v.shape == k.shape
        assert k.dtype == v.dtype == cfg.torch_dtype and k.get_device() == v.get_device()
        c.c = ee_kv_cache(_ptr(k), _ptr(v), c.num_blocks, cfg.block_size)
        return c


def make_batch(tokens: Optional[torch.Tensor], context_lens: torch.Tensor, block_tables: torch.Tensor,
               max_context: int, row_table: Optional[torch.Tensor] = None) -> ee_batch:
    B = int(context_lens.shape[0])
    b = ee_batch(B, _ptr(_i32(tokens)) if tokens is not None else None, _ptr(_i32(context_lens)),
                 _ptr(_i32(block_tables)), int(block_tables.shape[1]) if block_tables.dim() == 2 else 0, max_context,
                 _ptr(_i32(row_table)) if row_table is not None else None)
    b._keep = (tokens, context_lens, block_tables, row_table)   # the record only holds raw pointers: keep the tensors alive
    b.device = context_lens.get_device()
    assert all(t is None or t.get_device() == b.device for t in b._keep), "the tensors of a batch are on one device"
    return b


class Workspace:
    def __init__(self, desc: ee_model_desc, max_batch: int, max_context: int, device="cuda"):
        self.bytes = ee_workspace_bytes(desc, max_batch, max_context)
        if self.bytes == 0:
            raise EEError(EE_ERR_INVALID_ARG, ee_last_error())
        self.buf = torch.empty(self.bytes, dtype=torch.uint8, device=device)
        assert self.buf.data_ptr() % 256 == 0


EE_EXIT_NONE, EE_EXIT_BATCH, EE_EXIT_PER_SEQUENCE = 0, 1, 2


def ee_decode_iteration(model: DeviceModel, cache: PagedKV, batch: ee_batch, thresholds, forced_exit_layer,
                        use_exit_heads, out_tokens, out_exit_layer, out_batch_exit_layer, out_conf, out_hidden,
                        ws: Workspace):
    n = model.cfg.n_layers
    th = (C.c_float * n)(*([float(thresholds)] * n if isinstance(thresholds, (int, float)) else list(thresholds)))
    _check(lib().ee_decode_iteration(C.byref(model.c), C.byref(cache.c), C.byref(batch), th,
                                     _ptr(forced_exit_layer), int(use_exit_heads), _ptr(out_tokens),
                                     _ptr(out_exit_layer), _ptr(out_batch_exit_layer), _ptr(out_conf), _ptr(out_hidden),
                                     _ptr(ws.buf), ws.bytes, _stream()))


def ee_exit_check(model: DeviceModel, layer: int, hidden, threshold: float, forced_exit_layer, status, exit_layer,
                  n_exited, done_flag, batch_exit_layer, argmax, conf, ws: Workspace):
    _check(lib().ee_exit_check(C.byref(model.c), layer, _ptr(hidden), int(hidden.shape[0]), float(threshold),
                               _ptr(forced_exit_layer), _ptr(status), _ptr(exit_layer), _ptr(n_exited), _ptr(done_flag),
                               _ptr(batch_exit_layer), _ptr(argmax), _ptr(conf), _ptr(ws.buf), ws.bytes, _stream()))


def ee_noalloc_init():
    _check(lib().ee_noalloc_init())


def ee_exit_check_noalloc_bytes(desc: ee_model_desc, batch: int) -> int:
    return lib().ee_exit_check_noalloc_bytes(C.byref(desc), batch)


def ee_exit_check_noalloc(model: DeviceModel, layer: int, hidden, threshold: float, forced_exit_layer, status, exit_layer,
                          n_exited, done_flag, batch_exit_layer, argmax, conf):
    _check(lib().ee_exit_check_noalloc(C.byref(model.c), layer, _ptr(hidden), int(hidden.shape[0]), float(threshold),
                                       _ptr(forced_exit_layer), _ptr(status), _ptr(exit_layer), _ptr(n_exited),
                                       _ptr(done_flag), _ptr(batch_exit_layer), _ptr(argmax), _ptr(conf), _stream()))


def ee_kv_fill(model: DeviceModel, cache: PagedKV, batch: ee_batch, hidden, fill_from_layer, ws: Workspace):
    _check(lib().ee_kv_fill(C.byref(model.c), C.byref(cache.c), C.byref(batch), _ptr(hidden), _ptr(fill_from_layer),
                            _ptr(ws.buf), ws.bytes, _stream()))


def ee_paged_attention_decode(desc: ee_model_desc, cache: PagedKV, layer: int, q, batch: ee_batch, out,
                              ws: Optional[Workspace] = None):
    _check(lib().ee_paged_attention_decode(C.byref(desc), C.byref(cache.c), layer, _ptr(q), C.byref(batch), _ptr(out),
                                           _ptr(ws.buf) if ws else None, ws.bytes if ws else 0, _stream()))


# ---- 8-bit cache, rotary embedding on its own ------------------------------------------------------------
# One of these calls takes a few microseconds on the GPU at decode sizes, so the wrappers are kept short: a tensor is looked at once.
_KIND = {torch.float32: EE_FP32, torch.bfloat16: EE_BF16}


# The current device, and its current stream, which a call goes to: by torch's own short ways where it has them (0.2 us together, the public ones 1.3).
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _here(t: torch.Tensor, device: int) -> int:
    """The address of a contiguous tensor on the current device."""
    assert t.get_device() == device and t.is_contiguous(), "contiguous CUDA tensors of the current device"
    return t.data_ptr()


def _current_device(cache: "QuantKV", batch: ee_batch) -> int:
    """The current device, which is the cache's and the batch's."""
    device = _device()
    assert cache.device == device and getattr(batch, "device", device) == device, "a cache and a batch of the current device"
    return device


def _row_stride(t: torch.Tensor, rows: int, heads: int, dh: int, device: int) -> int:
    """The row stride of [rows][heads][channels] whose heads and channels are consecutive."""
    row, head, channel = t.stride()
    assert t.get_device() == device, "CUDA tensors of the current device"
    assert (channel == 1 or dh == 1) and (head == dh or heads == 1) or rows == 0, "heads and channels must be consecutive"
    return row if rows > 1 else heads * dh


def make_rotary_desc(head_dim: int, rotary_dim: Optional[int] = None, layout: str = "half", theta: float = 10000.0,
                     scaling: str = "plain", factor: float = 1.0, original_context: int = 1, turns=(1.0, 4.0),
                     amplitude: float = 1.0) -> ee_rotary_desc:
    layouts = {"half": EE_ROTARY_HALF, "interleaved": EE_ROTARY_INTERLEAVED}
    scalings = {"plain": EE_ROTARY_PLAIN, "linear": EE_ROTARY_LINEAR, "turns": EE_ROTARY_TURNS}
    return ee_rotary_desc(head_dim, head_dim if rotary_dim is None else rotary_dim, layouts[layout], scalings[scaling],
                          original_context, theta, factor, turns[0], turns[1], amplitude)


def ee_rotary_frequencies(desc: ee_rotary_desc, device="cuda") -> torch.Tensor:
    """The frequencies every later ee_rotary call with this desc takes (a new float64 tensor [rotary_dim / 2])."""
    freqs = torch.empty(max(0, desc.rotary_dim // 2), dtype=torch.float64, device=device)
    _check(lib().ee_rotary_frequencies(C.byref(desc), _here(freqs, _device()), _stream()))
    return freqs


def _rotary_side(x, y, rows, dh, device):
    shape = x.shape
    heads = shape[1]
    assert shape == (rows, heads, dh) and y.shape == shape and x.dtype == y.dtype
    return ee_rotary_rows(x.data_ptr(), y.data_ptr(), _row_stride(x, rows, heads, dh, device), _row_stride(y, rows, heads, dh, device), heads)


def ee_rotary(desc: ee_rotary_desc, freqs: torch.Tensor, positions: torch.Tensor, q: Optional[torch.Tensor],
              q_out: Optional[torch.Tensor], k: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
              transpose: bool = False):
    """Rows [rows][heads][head_dim] of any row stride; q_out may be q, k_out may be k."""
    assert freqs.dtype == torch.float64 and freqs.shape[0] == desc.rotary_dim // 2 and positions.dtype == torch.int32
    device, rows, dh = _device(), positions.shape[0], desc.head_dim
    assert q is None or k is None or q.dtype == k.dtype, "q, k and the results have one type"
    some = k if q is None else q
    _check(lib().ee_rotary(desc, _here(freqs, device), _here(positions, device), rows, EE_FP32 if some is None else _KIND[some.dtype],
                           None if q is None else _rotary_side(q, q_out, rows, dh, device),
                           None if k is None else _rotary_side(k, k_out, rows, dh, device), bool(transpose), _raw_stream(device)))


class QuantKV:
    """8-bit paged cache: k [n_layers][num_blocks][Hkv][16][dh], v [n_layers][num_blocks][Hkv][dh][16] (int8 or
    float8_e4m3fn) and scales [n_layers][num_blocks][Hkv][2] float."""

    def __init__(self, n_layers: int, num_blocks: int, n_kv_heads: int, head_dim: int, format: str = "int8", device="cuda"):
        t = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}[format]
        self._hold(torch.zeros((n_layers, num_blocks, n_kv_heads, 16, head_dim), dtype=torch.int8, device=device).view(t),
                   torch.zeros((n_layers, num_blocks, n_kv_heads, head_dim, 16), dtype=torch.int8, device=device).view(t),
                   torch.zeros((n_layers, num_blocks, n_kv_heads, 2), device=device))

    @classmethod
    def of(cls, k: torch.Tensor, v: torch.Tensor, scales: torch.Tensor) -> "QuantKV":
        """The record of a cache that is there already."""
        c = cls.__new__(cls)
        c._hold(k, v, scales)
        return c

    def _hold(self, k, v, scales):
        n, nb, h, bs, dh = k.shape
        assert k.dtype == v.dtype and k.dtype in (torch.int8, torch.float8_e4m3fn) and scales.dtype == torch.float32
        assert v.shape == (n, nb, h, dh, bs) and scales.shape == (n, nb, h, 2)
        self.k, self.v, self.scales, self.num_blocks, self.head = k, v, scales, nb, (h, dh)
        self.device = k.get_device()
        assert v.get_device() == self.device and scales.get_device() == self.device, "the pools of a cache are on one device"
        self.c = ee_quant_cache(_ptr(k), _ptr(v), _ptr(scales), n, nb, bs, h, dh,
                                EE_QUANT_INT8 if k.dtype == torch.int8 else EE_QUANT_E4M3)


class QuantWorkspace:
    """Scratch of ee_paged_attention_quant calls up to these sizes, or of ee_kv_quant_evict in place (`evicting`)."""

    def __init__(self, cache: QuantKV, n_heads: int, max_batch: int, max_context: int, with_weights: bool = False,
                 evicting: bool = False):
        L = lib()
        if evicting:
            self.bytes = L.ee_kv_quant_evict_bytes(C.byref(cache.c), max_batch, max_context)
        else:
            self.bytes = L.ee_paged_attention_quant_bytes(C.byref(cache.c), n_heads, max_batch, max_context, int(with_weights))
        if self.bytes == 0:
            raise EEError(EE_ERR_INVALID_ARG, ee_last_error())
        self.buf = torch.empty(self.bytes, dtype=torch.uint8, device=cache.k.device)
        assert self.buf.data_ptr() % 256 == 0


def ee_kv_quant_append(cache: QuantKV, layer: int, k: torch.Tensor, v: torch.Tensor, batch: ee_batch):
    """k, v [rows][Hkv][dh], float32 or bfloat16, any (even) row stride."""
    device, rows, (heads, dh) = _current_device(cache, batch), batch.batch, cache.head
    assert k.shape == (rows, heads, dh) and v.shape == k.shape and k.dtype == v.dtype, "k and v: rows of the batch, one type"
    _check(lib().ee_kv_quant_append(cache.c, layer, k.data_ptr(), _row_stride(k, rows, heads, dh, device), v.data_ptr(),
                                    _row_stride(v, rows, heads, dh, device), _KIND[k.dtype], batch, _raw_stream(device)))


def ee_kv_quant_read(cache: QuantKV, layer: int, batch: ee_batch, k: torch.Tensor, v: torch.Tensor):
    device = _current_device(cache, batch)
    assert k.shape == (batch.batch, *cache.head) and v.shape == k.shape and k.dtype == v.dtype, "k and v: rows of the batch, one type"
    _check(lib().ee_kv_quant_read(cache.c, layer, batch, _here(k, device), _here(v, device), _KIND[k.dtype], _raw_stream(device)))


def ee_paged_attention_quant(cache: QuantKV, layer: int, q: torch.Tensor, batch: ee_batch, out: torch.Tensor,
                             ws: Optional[QuantWorkspace] = None, weights_in: Optional[torch.Tensor] = None,
                             weights_out: Optional[torch.Tensor] = None):
    """q, out [rows][H][dh] float32; weights [rows][Hkv][pitch] float32."""
    device = _current_device(cache, batch)
    rows, heads, dh = q.shape
    assert out.shape == q.shape and rows == batch.batch and dh == cache.head[1]
    assert q.dtype == torch.float32 and out.dtype == torch.float32
    pitch = 0
    for w in (weights_in, weights_out):
        if w is not None:
            assert w.dtype == torch.float32 and w.shape[:2] == (rows, cache.head[0]) and pitch in (0, w.shape[2])
            pitch = w.shape[2]
    _check(lib().ee_paged_attention_quant(cache.c, layer, heads, _here(q, device), batch, _here(out, device),
                                          None if weights_in is None else _here(weights_in, device),
                                          None if weights_out is None else _here(weights_out, device), pitch,
                                          None if ws is None else _here(ws.buf, device), 0 if ws is None else ws.bytes, _raw_stream(device)))


def ee_kv_quant_evict(cache: QuantKV, layer: int, batch: ee_batch, weights_in: torch.Tensor, weights_out: Optional[torch.Tensor],
                      keep: int, recent: int, kept: torch.Tensor, out_lens: torch.Tensor, ws: Optional[QuantWorkspace] = None,
                      dst_tables: Optional[torch.Tensor] = None):
    """weights [B][Hkv][pitch] float32, kept [B][Hkv][keep] int32, out_lens [B] int32, dst_tables [B][blocks] int32."""
    device, head = _current_device(cache, batch), (batch.batch, cache.head[0])
    assert weights_in.dtype == torch.float32 and weights_in.shape[:2] == head
    assert weights_out is None or weights_out.dtype == torch.float32 and weights_out.shape[:2] == head
    assert kept.shape == (*head, keep) and out_lens.shape == head[:1] and kept.dtype == torch.int32 and out_lens.dtype == torch.int32
    assert dst_tables is None or dst_tables.shape[0] == head[0] and dst_tables.dtype == torch.int32
    _check(lib().ee_kv_quant_evict(cache.c, layer, batch, None if dst_tables is None else _here(dst_tables, device),
                                   0 if dst_tables is None else dst_tables.shape[1], _here(weights_in, device), weights_in.shape[2],
                                   None if weights_out is None else _here(weights_out, device),
                                   0 if weights_out is None else weights_out.shape[2], keep, recent, _here(kept, device),
                                   _here(out_lens, device), None if ws is None else _here(ws.buf, device), 0 if ws is None else ws.bytes,
                                   _raw_stream(device)))


# ---- several continuations of a prompt -------------------------------------------------------------------
class PagePool:
    """The references of a cache's blocks (int32 [num_blocks]), and the scratch of the calls that change them for up to max_rows rows.  Calls on one
    pool are ordered among themselves (one stream, or events between streams): they change the same counts."""

    def __init__(self, num_blocks: int, max_rows: int, device="cuda"):
        self._hold(torch.zeros(num_blocks, dtype=torch.int32, device=device), max_rows)

    @classmethod
    def of(cls, refs: torch.Tensor, max_rows: int) -> "PagePool":
        """The record of counts that are there already."""
        c = cls.__new__(cls)
        c._hold(refs, max_rows)
        return c

    def _hold(self, refs, max_rows):
        assert refs.dtype == torch.int32 and refs.dim() == 1
        self.refs, self.num_blocks, self.device = refs, refs.shape[0], refs.get_device()
        self.address = _ptr(refs)
        self.bytes = lib().ee_kv_pages_bytes(self.num_blocks, max_rows)
        if self.bytes == 0:
            raise EEError(EE_ERR_INVALID_ARG, ee_last_error())
        self.ws = torch.empty(self.bytes, dtype=torch.uint8, device=refs.device)
        assert self.ws.data_ptr() % 256 == 0


class PageTables:
    """Block tables [rows][max_blocks] and the cached positions [rows] of their rows, int32."""

    def __init__(self, block_tables: torch.Tensor, lens: torch.Tensor):
        assert block_tables.dtype == torch.int32 and lens.dtype == torch.int32 and block_tables.dim() == 2 and lens.shape == block_tables.shape[:1]
        assert block_tables.get_device() == lens.get_device(), "tables and lengths are on one device"
        self.block_tables, self.lens, self.rows, self.device = block_tables, lens, lens.shape[0], lens.get_device()
        self.c = ee_page_tables(_ptr(block_tables), _ptr(lens), *block_tables.shape)


def _pool_device(pool, tables, more=None) -> int:
    device = _device()
    assert (pool is None or pool.device == device) and (tables is None or tables.device == device) and (more is None or more.device == device), \
        "a pool and tables of the current device"
    return device


def _int32s(t: torch.Tensor, shape, device: int) -> int:
    assert t.dtype is torch.int32 and t.shape == shape, "int32 of the call's sizes"
    assert t.get_device() == device and t.is_contiguous(), "contiguous CUDA tensors of the current device"
    return t.data_ptr()


def ee_kv_pages_fork(pool: PagePool, src: PageTables, parents: torch.Tensor, dst: PageTables, release: bool = False):
    """Row m of dst becomes row parents[m] of src; with release the rows of src give up their blocks."""
    device = _pool_device(pool, src, dst)
    _check(lib().ee_kv_pages_fork(pool.address, pool.num_blocks, src.c, _int32s(parents, (dst.rows,), device), dst.c, bool(release), _raw_stream(device)))


def ee_kv_pages_release(pool: PagePool, tables: PageTables):
    device = _pool_device(pool, tables)
    _check(lib().ee_kv_pages_release(pool.address, pool.num_blocks, tables.c, _raw_stream(device)))


def ee_kv_pages_grow(pool: PagePool, tables: PageTables, new_lens: torch.Tensor, moves: torch.Tensor, missing: torch.Tensor):
    """new_lens [rows], moves [rows][2], missing [1], int32."""
    device, rows = _pool_device(pool, tables), tables.rows
    _check(lib().ee_kv_pages_grow(pool.address, pool.num_blocks, tables.c, _int32s(new_lens, (rows,), device), _int32s(moves, (rows, 2), device),
                                  _int32s(missing, (1,), device), pool.ws.data_ptr(), pool.bytes, _raw_stream(device)))


def ee_kv_pages_compact(pool: PagePool, tables: Optional[PageTables], remap: torch.Tensor, moves: torch.Tensor, n_moves: torch.Tensor):
    """remap [num_blocks], moves [num_blocks][2], n_moves [1], int32."""
    device, n = _pool_device(pool, tables), pool.num_blocks
    _check(lib().ee_kv_pages_compact(pool.address, n, None if tables is None else tables.c, _int32s(remap, (n,), device), _int32s(moves, (n, 2), device),
                                     _int32s(n_moves, (1,), device), pool.ws.data_ptr(), pool.bytes, _raw_stream(device)))


def ee_kv_pages_shared(tables: PageTables, first_row: torch.Tensor, shared_blocks: torch.Tensor):
    """first_row [groups + 1], shared_blocks [groups], int32."""
    device, n = _pool_device(None, tables), shared_blocks.shape[0]
    _check(lib().ee_kv_pages_shared(tables.c, _int32s(first_row, (n + 1,), device), n, _int32s(shared_blocks, (n,), device), _raw_stream(device)))


def ee_kv_copy(desc: ee_model_desc, cache: PagedKV, moves: torch.Tensor, count: Optional[torch.Tensor] = None):
    """moves [n][2] int32; count [1] int32: only the first of them."""
    device, n = _device(), moves.shape[0]
    assert cache.k.get_device() == device, "a cache of the current device"
    _check(lib().ee_kv_copy(desc, cache.c, _int32s(moves, (n, 2), device), n, None if count is None else _int32s(count, (1,), device), _raw_stream(device)))


def ee_kv_quant_copy(cache: QuantKV, moves: torch.Tensor, count: Optional[torch.Tensor] = None):
    device, n = _device(), moves.shape[0]
    assert cache.device == device, "a cache of the current device"
    _check(lib().ee_kv_quant_copy(cache.c, _int32s(moves, (n, 2), device), n, None if count is None else _int32s(count, (1,), device), _raw_stream(device)))


class BeamWorkspace:
    """Scratch of ee_beam_select calls of these sizes."""

    def __init__(self, groups: int, beams: int, vocab: int, n_out: int, device="cuda"):
        self.bytes = lib().ee_beam_select_bytes(groups, beams, vocab, n_out)
        if self.bytes == 0:
            raise EEError(EE_ERR_INVALID_ARG, ee_last_error())
        self.buf = torch.empty(self.bytes, dtype=torch.uint8, device=device)
        self.address, self.device = self.buf.data_ptr(), self.buf.get_device()
        assert self.address % 256 == 0


def ee_beam_select(logits: torch.Tensor, scores: torch.Tensor, beams: int, tokens: torch.Tensor, parents: torch.Tensor, scores_out: torch.Tensor,
                   ws: BeamWorkspace, finished: Optional[torch.Tensor] = None, finished_out: Optional[torch.Tensor] = None, end_token: int = -1):
    """logits [groups * beams][vocab] float32 or bfloat16, any row stride; scores [groups * beams] float32; finished [groups * beams] int32; the results
    [groups * n_out] (or [groups][n_out])."""
    device, (rows, vocab), (row_stride, stride) = _device(), logits.shape, logits.stride()
    groups, total = rows // beams if beams > 0 else 0, tokens.numel()
    n_out = total // groups if groups else 1
    assert beams > 0 and rows == groups * beams == scores.numel() and total == groups * n_out == parents.numel() == scores_out.numel(), "rows of whole groups"
    assert scores.dtype is scores_out.dtype is torch.float32 and tokens.dtype is parents.dtype is torch.int32
    assert logits.get_device() == device == ws.device and (stride == 1 or vocab == 1), "rows of consecutive values, and a workspace, on the current device"
    assert device == scores.get_device() == tokens.get_device() == parents.get_device() == scores_out.get_device() and scores.is_contiguous() and tokens.is_contiguous() \
        and parents.is_contiguous() and scores_out.is_contiguous(), "contiguous CUDA tensors of the current device"
    assert finished is None or finished.numel() == rows and finished.dtype is torch.int32
    assert finished_out is None or finished_out.numel() == total and finished_out.dtype is torch.int32
    _check(lib().ee_beam_select(logits.data_ptr(), row_stride if rows > 1 else vocab, _KIND[logits.dtype], scores.data_ptr(),
                                None if finished is None else _here(finished, device), groups, beams, vocab, n_out, end_token,
                                tokens.data_ptr(), parents.data_ptr(), scores_out.data_ptr(),
                                None if finished_out is None else _here(finished_out, device), ws.address, ws.bytes, _raw_stream(device)))


def ee_reorder_rows(x: torch.Tensor, parents: torch.Tensor, out: torch.Tensor):
    """out[m] = x[parents[m]] of any type, rows of consecutive values at any row stride."""
    device, rows, shape, out_shape = _device(), parents.numel(), x.shape, out.shape
    assert x.dtype is out.dtype and (shape == out_shape or shape[1:] == out_shape[1:]) and out_shape[0] == rows and parents.dtype is torch.int32
    assert x.get_device() == device and out.get_device() == device, "CUDA tensors of the current device"
    row = out.nbytes // rows if rows else 0
    x_stride = out_stride = row
    if not x.is_contiguous():
        assert x[0].is_contiguous(), "rows of consecutive values"
        x_stride = x.stride(0) * x.element_size() if shape[0] > 1 else row
    if not out.is_contiguous():
        assert out[0].is_contiguous(), "rows of consecutive values"
        out_stride = out.stride(0) * out.element_size() if rows > 1 else row
    _check(lib().ee_reorder_rows(x.data_ptr(), x_stride, shape[0], _here(parents, device), rows, row, out.data_ptr(), out_stride, _raw_stream(device)))


def make_prefix_groups(first_row: torch.Tensor, shared_blocks: torch.Tensor, max_shared: int) -> ee_prefix_groups:
    """first_row [groups + 1], shared_blocks [groups], int32; max_shared bounds the latter."""
    assert first_row.shape == (shared_blocks.shape[0] + 1,)
    g = ee_prefix_groups(shared_blocks.shape[0], _ptr(_i32(first_row)), _ptr(_i32(shared_blocks)), max_shared)
    g._keep = (first_row, shared_blocks)   # the record only holds raw pointers
    g.device = first_row.get_device()
    assert shared_blocks.get_device() == g.device, "the tensors of groups are on one device"
    return g


class SharedWorkspace:
    """Scratch of ee_paged_attention_shared calls up to these sizes."""

    def __init__(self, desc: ee_model_desc, n_heads: int, max_batch: int, max_groups: int, max_context: int, device="cuda"):
        self.bytes = lib().ee_paged_attention_shared_bytes(desc, n_heads, max_batch, max_groups, max_context)
        if self.bytes == 0:
            raise EEError(EE_ERR_INVALID_ARG, ee_last_error())
        self.buf = torch.empty(self.bytes, dtype=torch.uint8, device=device)
        self.address, self.device = self.buf.data_ptr(), self.buf.get_device()
        assert self.address % 256 == 0


def ee_paged_attention_shared(desc: ee_model_desc, cache: PagedKV, layer: int, q: torch.Tensor, batch: ee_batch, groups: ee_prefix_groups,
                              out: torch.Tensor, ws: SharedWorkspace):
    """q, out [rows][n_heads][dh] float32; the cache has desc.n_heads K/V heads."""
    device = _device()
    assert cache.k.get_device() == device == getattr(batch, "device", device) and device == getattr(groups, "device", device) == ws.device, \
        "cache, batch, groups and workspace of the current device"
    rows, heads, dh = q.shape
    assert out.shape == q.shape and rows == batch.batch and dh == desc.head_dim and q.dtype == torch.float32 and out.dtype == torch.float32
    _check(lib().ee_paged_attention_shared(desc, cache.c, layer, heads, _here(q, device), batch, groups, _here(out, device), ws.address, ws.bytes,
                                           _raw_stream(device)))


def ee_profile_enable(on: bool):
    _check(lib().ee_profile_enable(int(bool(on))))


def ee_profile_read(max_records: int = 1 << 20):
    """Returns a list of (class name, layer, milliseconds) for every kernel enqueued since the last read."""
    cls = (C.c_int32 * max_records)()
    lay = (C.c_int32 * max_records)()
    ms = (C.c_float * max_records)()
    n = lib().ee_profile_read(cls, lay, ms, max_records)
    if n < 0:
        raise EEError(n, ee_last_error())
    return [(KERNEL_CLASSES[cls[i]], lay[i], ms[i]) for i in range(n)]


def ee_calibration_copy(src: torch.Tensor, dst: torch.Tensor):
    assert src.dtype == torch.float32 and dst.dtype == torch.float32 and src.numel() == dst.numel()
    _check(lib().ee_calibration_copy(_ptr(src), _ptr(dst), src.numel(), _stream()))


def ee_calibration_read(src: torch.Tensor, sink: torch.Tensor, workgroups: int):
    _check(lib().ee_calibration_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink), workgroups, _stream()))


def ee_calibration_mfma(workgroups: int, iterations: int, sink: torch.Tensor):
    assert sink.dtype == torch.float32 and sink.numel() >= 256
    _check(lib().ee_calibration_mfma(workgroups, iterations, _ptr(sink), _stream()))


def ee_calibration_intake(own: torch.Tensor, common: torch.Tensor, workgroups: int, loads_in_flight: int, pairs: bool,
                          sink: torch.Tensor):
    _check(lib().ee_calibration_intake(_ptr(own), own.numel() * own.element_size(), _ptr(common),
                                       common.numel() * common.element_size(), workgroups, loads_in_flight, int(pairs),
                                       _ptr(sink), _stream()))


def ee_calibration_mfma_tile(workgroups: int, steps: int, lds_fragment_reads: int, sink: torch.Tensor):
    assert sink.dtype == torch.float32 and sink.numel() >= 256
    _check(lib().ee_calibration_mfma_tile(workgroups, steps, lds_fragment_reads, _ptr(sink), _stream()))
