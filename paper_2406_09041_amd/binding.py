"""Thin ctypes binding over libmes.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels.  PyTorch is used for device
memory (tensors own every buffer) and for the current HIP stream.  There is no CPU
fallback: if libmes.so is missing the import fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("MES_LIBRARY") or os.path.join(_HERE, "libmes.so")   # MES_LIBRARY: another build of the same library

MES_OK = 0
GRID_SYM, GRID_EQ1 = 0, 1
STEP_GIVEN, STEP_MAXABS, STEP_MEANABS = 0, 1, 2
MAX_EXPERTS = 64

KV_BF16, KV_E4M3, KV_E4M3_BLOCKS = 0, 1, 3
KV_BLOCK, LEAST_EXPONENT = 16, 10      # tokens of a block; the least exponent byte that is written
ROTARY_HALVES, ROTARY_PAIRS = 0, 1
SCALINGS = {None: 0, "linear": 1, "base": 2, "bands": 3}
MAX_SEQS = 2048
SHORT_PROMPT = 704          # keys, 11 tiles of 64: the library never shares out rows that see no more, and needs no workspace for them

STATUS_NAMES = {0: "MES_OK", 1: "MES_ERR_NULL", 2: "MES_ERR_SHAPE", 3: "MES_ERR_BITS", 4: "MES_ERR_SALIENT",
                5: "MES_ERR_SEGMENTS", 6: "MES_ERR_ALIGN", 7: "MES_ERR_WORKSPACE", 8: "MES_ERR_DEVICE", 9: "MES_ERR_PAGES"}

EXPORTS = ["mes_base_bytes", "mes_codes_bytes", "mes_salient_bytes", "mes_pack_workspace_bytes",
           "mes_select_workspace_bytes", "mes_linear_workspace_bytes", "mes_last_error", "mes_layout_version",
           "mes_pack_base", "mes_unpack_base", "mes_select_salient", "mes_pack_delta", "mes_unpack_delta",
           "mes_delta_linear", "mes_linear_multi_workspace_bytes",
           "mes_delta_linear_multi", "mes_time_next_call", "mes_copy_probe", "mes_pool_slot_bytes", "mes_pool_create",
           "mes_pool_destroy", "mes_pool_register", "mes_pool_acquire", "mes_pool_slot_of", "mes_pool_stats",
           "mes_pool_slot_layout", "mes_pool_multi_slot_bytes", "mes_pool_create_multi", "mes_pool_linear_offset",
           "mes_pool_register_blob", "mes_pool_acquire_multi", "mes_pool_prefetch", "mes_pool_prefetched",
           "mes_gated_workspace_bytes", "mes_delta_linear_gated",
           "mes_step_grad_workspace_bytes", "mes_step_grad", "mes_step_adamw", "mes_noalloc_scratch_bytes",
           "mes_delta_linear_noalloc", "mes_long_segment_tokens",
           "mes_kv_append", "mes_kv_append_fresh", "mes_attn_prompt", "mes_attn_prompt_workspace_bytes", "mes_attn_extend", "mes_attn_decode_workspace_bytes", "mes_attn_decode",
           "mes_kv_append_angles", "mes_rotary_table", "mes_rotary", "mes_kv_read", "mes_kv_copy_pages", "mes_pages_create", "mes_pages_destroy", "mes_pages_grow", "mes_pages_fork", "mes_pages_free",
           "mes_pages_compact", "mes_pages_table", "mes_pages_length", "mes_pages_unused"]


class MesError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class mes_delta(ctypes.Structure):
    _fields_ = [("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32), ("k", ctypes.c_int32),
                ("bits", ctypes.c_int32), ("grid", ctypes.c_int32), ("layout_version", ctypes.c_int32),
                ("codes", ctypes.c_void_p), ("step", ctypes.c_void_p), ("salient", ctypes.c_void_p),
                ("salient_idx", ctypes.c_void_p)]


class mes_linear(ctypes.Structure):
    _fields_ = [("w_base_tiled", ctypes.c_void_p), ("experts", ctypes.POINTER(mes_delta)), ("y", ctypes.c_void_p)]


class mes_kv(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "n_pages", "page_tokens", "n_kv_heads", "head_dim", "dtype")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class mes_angles(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("n_positions", "dims", "layout")]


class mes_seqs(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("table_pages", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("q_offsets", "kv_len", "page_table")]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(LIB_PATH)
    c_int, c_sz, vp = ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p
    lib.mes_base_bytes.restype = c_sz
    lib.mes_base_bytes.argtypes = [c_int, c_int]
    lib.mes_codes_bytes.restype = c_sz
    lib.mes_codes_bytes.argtypes = [c_int, c_int, c_int]
    lib.mes_salient_bytes.restype = c_sz
    lib.mes_salient_bytes.argtypes = [c_int, c_int]
    lib.mes_pack_workspace_bytes.restype = c_sz
    lib.mes_pack_workspace_bytes.argtypes = []
    lib.mes_select_workspace_bytes.restype = c_sz
    lib.mes_select_workspace_bytes.argtypes = [c_int, c_int, c_int]
    lib.mes_linear_workspace_bytes.restype = c_sz
    lib.mes_linear_workspace_bytes.argtypes = [c_int, c_int, c_int]
    lib.mes_last_error.restype = ctypes.c_char_p
    lib.mes_last_error.argtypes = []
    lib.mes_layout_version.restype = c_int
    lib.mes_layout_version.argtypes = []
    lib.mes_pack_base.restype = c_int
    lib.mes_pack_base.argtypes = [vp, c_int, c_int, vp, vp]
    lib.mes_unpack_base.restype = c_int
    lib.mes_unpack_base.argtypes = [vp, c_int, c_int, vp, vp]
    lib.mes_select_salient.restype = c_int
    lib.mes_select_salient.argtypes = [vp, vp, c_int, c_int, c_int, c_int, c_int, c_int, c_int, vp, vp, vp, c_sz, vp]
    lib.mes_pack_delta.restype = c_int
    lib.mes_pack_delta.argtypes = [vp, c_int, c_int, vp, c_int, c_int, c_int, c_int, vp, vp, vp, vp, vp, c_sz, vp]
    lib.mes_unpack_delta.restype = c_int
    lib.mes_unpack_delta.argtypes = [ctypes.POINTER(mes_delta), vp, vp, vp]
    lib.mes_delta_linear.restype = c_int
    lib.mes_delta_linear.argtypes = [vp, ctypes.POINTER(mes_delta), c_int, vp, c_int,
                                     ctypes.POINTER(ctypes.c_int32), vp, vp, c_sz, vp]
    lib.mes_long_segment_tokens.restype = c_int
    lib.mes_long_segment_tokens.argtypes = []
    lib.mes_noalloc_scratch_bytes.restype = c_sz
    lib.mes_noalloc_scratch_bytes.argtypes = []
    lib.mes_delta_linear_noalloc.restype = c_int
    lib.mes_delta_linear_noalloc.argtypes = [vp, ctypes.POINTER(mes_delta), c_int, vp, c_int,
                                             ctypes.POINTER(ctypes.c_int32), vp, vp]
    lib.mes_linear_multi_workspace_bytes.restype = c_sz
    lib.mes_linear_multi_workspace_bytes.argtypes = [c_int, ctypes.POINTER(ctypes.c_int32), c_int, c_int]
    lib.mes_delta_linear_multi.restype = c_int
    lib.mes_delta_linear_multi.argtypes = [ctypes.POINTER(mes_linear), c_int, c_int, vp, c_int,
                                           ctypes.POINTER(ctypes.c_int32), vp, c_sz, vp]
    lib.mes_time_next_call.restype = c_int
    lib.mes_time_next_call.argtypes = [vp, vp]
    lib.mes_step_grad_workspace_bytes.restype = c_sz
    lib.mes_step_grad_workspace_bytes.argtypes = [c_int, c_int, c_int]
    lib.mes_step_grad.restype = c_int
    lib.mes_step_grad.argtypes = [vp, c_int, c_int, vp, c_int, c_int, c_int, vp, vp, c_int, vp, vp, vp, c_sz, vp]
    lib.mes_step_adamw.restype = c_int
    lib.mes_step_adamw.argtypes = [vp, vp, vp, vp, c_int, c_int, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                   ctypes.c_float, ctypes.c_float, vp]
    lib.mes_copy_probe.restype = c_int
    lib.mes_copy_probe.argtypes = [vp, vp, c_sz, vp]
    lib.mes_pool_slot_bytes.restype = c_sz
    lib.mes_pool_slot_bytes.argtypes = [c_int, c_int, c_int, c_int]
    lib.mes_pool_create.restype = c_int
    lib.mes_pool_create.argtypes = [c_int, c_int, c_int, c_int, c_int, c_int, c_int, vp, c_sz, c_int, ctypes.POINTER(vp)]
    lib.mes_pool_destroy.restype = None
    lib.mes_pool_destroy.argtypes = [vp]
    lib.mes_pool_register.restype = c_int
    lib.mes_pool_register.argtypes = [vp, c_int, vp, vp, vp, vp]
    lib.mes_pool_acquire.restype = c_int
    lib.mes_pool_acquire.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), c_int, ctypes.POINTER(mes_delta), vp, vp]
    lib.mes_pool_slot_of.restype = c_int
    lib.mes_pool_slot_of.argtypes = [vp, c_int]
    lib.mes_gated_workspace_bytes.restype = c_sz
    lib.mes_gated_workspace_bytes.argtypes = [c_int, c_int, c_int]
    lib.mes_delta_linear_gated.restype = c_int
    lib.mes_delta_linear_gated.argtypes = [vp, ctypes.POINTER(mes_delta), vp, ctypes.POINTER(mes_delta), c_int, vp, c_int,
                                           ctypes.POINTER(ctypes.c_int32), vp, vp, c_sz, vp]
    i32p = ctypes.POINTER(ctypes.c_int32)
    lib.mes_pool_slot_layout.restype = c_sz
    lib.mes_pool_slot_layout.argtypes = [c_int, c_int, c_int, c_int, ctypes.POINTER(c_sz)]
    lib.mes_pool_multi_slot_bytes.restype = c_sz
    lib.mes_pool_multi_slot_bytes.argtypes = [c_int, i32p, i32p, i32p, c_int]
    lib.mes_pool_create_multi.restype = c_int
    lib.mes_pool_create_multi.argtypes = [c_int, i32p, i32p, i32p, c_int, c_int, c_int, c_int, vp, c_sz, c_int, ctypes.POINTER(vp)]
    lib.mes_pool_linear_offset.restype = c_sz
    lib.mes_pool_linear_offset.argtypes = [vp, c_int]
    lib.mes_pool_register_blob.restype = c_int
    lib.mes_pool_register_blob.argtypes = [vp, c_int, vp]
    lib.mes_pool_acquire_multi.restype = c_int
    lib.mes_pool_acquire_multi.argtypes = [vp, i32p, c_int, ctypes.POINTER(mes_delta), vp, vp]
    lib.mes_pool_prefetch.restype = c_int
    lib.mes_pool_prefetch.argtypes = [vp, i32p, c_int, ctypes.POINTER(c_int), vp]
    lib.mes_pool_prefetched.restype = ctypes.c_uint64
    lib.mes_pool_prefetched.argtypes = [vp]
    lib.mes_pool_stats.restype = c_int
    lib.mes_pool_stats.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64)]
    kvp, sqp, fl = ctypes.POINTER(mes_kv), ctypes.POINTER(mes_seqs), ctypes.c_float
    lib.mes_kv_append.restype = lib.mes_kv_append_fresh.restype = c_int
    lib.mes_kv_append.argtypes = lib.mes_kv_append_fresh.argtypes = [kvp, c_int, sqp, vp, vp, vp, c_int, c_int, c_int, c_int, c_int, vp, c_int, vp, c_int, vp]
    anp, db = ctypes.POINTER(mes_angles), ctypes.c_double
    lib.mes_kv_append_angles.restype = lib.mes_rotary_table.restype = lib.mes_rotary.restype = lib.mes_kv_read.restype = c_int
    lib.mes_kv_append_angles.argtypes = [kvp, c_int, sqp, vp, vp, vp, c_int, c_int, c_int, c_int, c_int, anp, vp, c_int, c_int, vp]
    lib.mes_rotary_table.argtypes = [vp, c_int, c_int, db, c_int, db, c_int, db, db, db, vp]
    lib.mes_rotary.argtypes = [anp, vp, vp, vp, c_int, c_int, c_int, c_int, c_int, c_int, c_int, c_int, vp, c_int, vp, c_int, c_int, vp]
    lib.mes_kv_read.argtypes = [kvp, c_int, sqp, c_int, vp, vp, c_int, c_int, c_int, vp]
    lib.mes_attn_prompt.restype = c_int
    lib.mes_attn_prompt.argtypes = [vp, vp, vp, c_int, c_int, vp, c_int, c_int, c_int, c_int, c_int, c_int, fl, vp, c_int, vp, c_sz, vp]
    lib.mes_attn_prompt_workspace_bytes.restype = c_sz
    lib.mes_attn_prompt_workspace_bytes.argtypes = [c_int] * 5
    lib.mes_attn_extend.restype = c_int
    lib.mes_attn_extend.argtypes = [kvp, c_int, sqp, vp, c_int, c_int, c_int, fl, vp, c_int, vp, c_sz, vp]
    lib.mes_attn_decode_workspace_bytes.restype = c_sz
    lib.mes_attn_decode_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int]
    lib.mes_attn_decode.restype = c_int
    lib.mes_attn_decode.argtypes = [kvp, c_int, sqp, vp, c_int, c_int, c_int, i32p, i32p, fl, vp, c_int, vp, c_sz, vp]
    lib.mes_kv_copy_pages.restype = c_int
    lib.mes_kv_copy_pages.argtypes = [kvp, i32p, i32p, c_int, vp]
    lib.mes_pages_create.restype = c_int
    lib.mes_pages_create.argtypes = [c_int, c_int, c_int, c_int, ctypes.POINTER(vp)]
    lib.mes_pages_destroy.restype = None
    lib.mes_pages_destroy.argtypes = [vp]
    lib.mes_pages_grow.restype = c_int
    lib.mes_pages_grow.argtypes = [vp, i32p, i32p, c_int, i32p, i32p, ctypes.POINTER(c_int)]
    lib.mes_pages_fork.restype = c_int
    lib.mes_pages_fork.argtypes = [vp, c_int, c_int, c_int]
    lib.mes_pages_free.restype = c_int
    lib.mes_pages_free.argtypes = [vp, c_int]
    lib.mes_pages_compact.restype = c_int
    lib.mes_pages_compact.argtypes = [vp, i32p, i32p, ctypes.POINTER(c_int)]
    lib.mes_pages_table.restype = c_int
    lib.mes_pages_table.argtypes = [vp, i32p, c_int, vp, c_int, vp]
    lib.mes_pages_length.restype = c_int
    lib.mes_pages_length.argtypes = [vp, c_int]
    lib.mes_pages_unused.restype = c_int
    lib.mes_pages_unused.argtypes = [vp]
    return lib


lib = _load()


def _check(status: int) -> None:
    if status != MES_OK:
        raise MesError(status, lib.mes_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def base_bytes(d_in, d_out): return lib.mes_base_bytes(d_in, d_out)
def codes_bytes(d_in, d_out, bits): return lib.mes_codes_bytes(d_in, d_out, bits)
def salient_bytes(d_out, k): return lib.mes_salient_bytes(d_out, k)
def linear_workspace_bytes(d_in, d_out, max_tokens): return lib.mes_linear_workspace_bytes(d_in, d_out, max_tokens)


def mes_pack_base(w: torch.Tensor) -> torch.Tensor:
    """w: bf16 [d_out, d_in] on the GPU -> tiled base (uint8 tensor of mes_base_bytes)."""
    assert w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous()
    d_out, d_in = w.shape
    out = torch.empty(base_bytes(d_in, d_out), dtype=torch.uint8, device=w.device)
    _check(lib.mes_pack_base(_ptr(w), d_in, d_out, _ptr(out), _stream(w.device)))
    return out


def mes_copy_probe(dst: torch.Tensor, src: torch.Tensor) -> None:
    """Plain copy kernel of known traffic (src.nbytes read, as many written); see mes_copy_probe in mes_bench.h."""
    assert dst.is_cuda and src.is_cuda and dst.is_contiguous() and src.is_contiguous() and dst.nbytes == src.nbytes
    _check(lib.mes_copy_probe(_ptr(dst), _ptr(src), src.nbytes, _stream(src.device)))


def mes_unpack_base(w_tiled: torch.Tensor, d_in: int, d_out: int) -> torch.Tensor:
    out = torch.empty((d_out, d_in), dtype=torch.bfloat16, device=w_tiled.device)
    _check(lib.mes_unpack_base(_ptr(w_tiled), d_in, d_out, _ptr(out), _stream(w_tiled.device)))
    return out


@dataclass
class PackedDelta:
    """Device buffers of one expert's compressed delta (see include/mes.h for the layouts)."""
    d_in: int
    d_out: int
    k: int
    bits: int
    grid: int
    codes: torch.Tensor                  # uint8 [mes_codes_bytes]
    step: torch.Tensor                   # fp32 [d_out]
    salient: Optional[torch.Tensor]      # uint8 [mes_salient_bytes] or None
    salient_idx: Optional[torch.Tensor]  # int32 [k] or None

    def descriptor(self) -> mes_delta:
        return mes_delta(self.d_in, self.d_out, self.k, self.bits, self.grid, lib.mes_layout_version(),
                         self.codes.data_ptr(), self.step.data_ptr(),
                         self.salient.data_ptr() if self.salient is not None else None,
                         self.salient_idx.data_ptr() if self.salient_idx is not None else None)


def mes_pack_delta(delta: torch.Tensor, salient_idx: Optional[torch.Tensor], bits: int, grid: int = GRID_SYM,
                   step_policy: int = STEP_MAXABS, step_in: Optional[torch.Tensor] = None) -> PackedDelta:
    """delta: fp32 [d_out, d_in] on the GPU; salient_idx: int32 [k] ascending (any device) or None."""
    assert delta.dtype == torch.float32 and delta.is_cuda and delta.is_contiguous()
    dev = delta.device
    d_out, d_in = delta.shape
    k = 0 if salient_idx is None else int(salient_idx.numel())
    sidx = None if k == 0 else salient_idx.to(device=dev, dtype=torch.int32).contiguous()
    codes = torch.empty(max(codes_bytes(d_in, d_out, bits), 16), dtype=torch.uint8, device=dev)
    step = torch.empty(d_out, dtype=torch.float32, device=dev)
    sal = None if k == 0 else torch.empty(salient_bytes(d_out, k), dtype=torch.uint8, device=dev)
    ws = torch.empty(lib.mes_pack_workspace_bytes(), dtype=torch.uint8, device=dev)
    if step_in is not None:
        step_in = step_in.to(device=dev, dtype=torch.float32).contiguous()
    _check(lib.mes_pack_delta(_ptr(delta), d_in, d_out, _ptr(sidx), k, bits, grid, step_policy, _ptr(step_in),
                              _ptr(codes), _ptr(step), _ptr(sal), _ptr(ws), ws.numel(), _stream(dev)))
    return PackedDelta(d_in, d_out, k, bits, grid, codes, step, sal, sidx)


def mes_unpack_delta(p: PackedDelta, want_codes: bool = True, want_delta: bool = True):
    dev = p.codes.device
    dh = torch.empty((p.d_out, p.d_in), dtype=torch.float32, device=dev) if want_delta else None
    cd = torch.empty((p.d_out, p.d_in), dtype=torch.uint8, device=dev) if want_codes else None
    desc = p.descriptor()
    _check(lib.mes_unpack_delta(ctypes.byref(desc), _ptr(dh), _ptr(cd), _stream(dev)))
    return dh, cd


def mes_select_salient(delta: torch.Tensor, x_calib: torch.Tensor, bits: int, grid: int, k: int,
                       step_policy: int = STEP_MAXABS, want_scores: bool = False):
    """Eq. 2 selection.  Returns idx int32 [k] ascending (and the fp64 scores [d_in] if asked)."""
    assert delta.dtype == torch.float32 and x_calib.dtype == torch.float32 and delta.is_cuda and x_calib.is_cuda
    dev = delta.device
    d_out, d_in = delta.shape
    n = x_calib.shape[0]
    idx = torch.empty(max(k, 1), dtype=torch.int32, device=dev)
    score = torch.empty(d_in, dtype=torch.float64, device=dev) if want_scores else None
    ws = torch.empty(max(lib.mes_select_workspace_bytes(n, d_in, d_out), 16), dtype=torch.uint8, device=dev)
    _check(lib.mes_select_salient(_ptr(delta.contiguous()), _ptr(x_calib.contiguous()), n, d_in, d_out, bits, grid,
                                  step_policy, k, _ptr(idx), _ptr(score), _ptr(ws), ws.numel(), _stream(dev)))
    idx = idx[:k]
    return (idx, score) if want_scores else idx


class StepGrad:
    """Marshalled arguments of mes_step_grad for one delta matrix (workspace and outputs allocated once)."""

    def __init__(self, delta: torch.Tensor, salient_idx: Optional[torch.Tensor], bits: int, grid: int = GRID_SYM,
                 max_tokens: int = 512):
        assert delta.dtype == torch.float32 and delta.is_cuda and delta.is_contiguous()
        self.delta, self.bits, self.grid = delta, bits, grid
        self.d_out, self.d_in = delta.shape
        self.k = 0 if salient_idx is None else int(salient_idx.numel())
        self.sidx = None if self.k == 0 else salient_idx.to(device=delta.device, dtype=torch.int32).contiguous()
        self.max_tokens = max_tokens
        n = max(lib.mes_step_grad_workspace_bytes(self.d_in, self.d_out, max_tokens), 16)
        self.ws = torch.empty(n, dtype=torch.uint8, device=delta.device)
        self.loss = torch.empty(self.d_out, dtype=torch.float32, device=delta.device)
        self.grad = torch.empty(self.d_out, dtype=torch.float32, device=delta.device)

    def __call__(self, step: torch.Tensor, x: torch.Tensor):
        """step fp32 [d_out], x bf16 [n_tokens, d_in] -> (loss [d_out], grad [d_out]), overwritten by the next call."""
        assert step.dtype == torch.float32 and x.dtype == torch.bfloat16 and x.shape[0] <= self.max_tokens
        _check(lib.mes_step_grad(_ptr(self.delta), self.d_in, self.d_out, _ptr(self.sidx), self.k, self.bits, self.grid,
                                 _ptr(step), _ptr(x), x.shape[0], _ptr(self.loss), _ptr(self.grad), _ptr(self.ws),
                                 self.ws.numel(), _stream(self.delta.device)))
        return self.loss, self.grad


def mes_step_adamw(step: torch.Tensor, grad: torch.Tensor, m: torch.Tensor, v: torch.Tensor, t: int, lr: float,
                   beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01) -> None:
    """One in-place AdamW update of the step vector (and of the moments m, v)."""
    _check(lib.mes_step_adamw(_ptr(step), _ptr(grad), _ptr(m), _ptr(v), step.numel(), t, lr, beta1, beta2, eps,
                              weight_decay, _stream(step.device)))


def make_workspace(d_in: int, d_out: int, max_tokens: int, device) -> torch.Tensor:
    """Allocates a mes_delta_linear workspace (scratch: its contents do not matter)."""
    n = max(linear_workspace_bytes(d_in, d_out, max_tokens), 16)
    return torch.empty(n, dtype=torch.uint8, device=device)


class DeltaLinear:
    """Marshalled arguments of mes_delta_linear for one layer (descriptor array built once)."""

    def __init__(self, w_base_tiled: torch.Tensor, experts: Sequence[PackedDelta], max_tokens: int = 64,
                 workspace: Optional[torch.Tensor] = None):
        self.w = w_base_tiled
        self.experts = list(experts)
        self.E = len(self.experts)
        self.d_in, self.d_out = self.experts[0].d_in, self.experts[0].d_out
        self.desc = (mes_delta * self.E)(*[e.descriptor() for e in self.experts])
        self.ws = workspace if workspace is not None else make_workspace(self.d_in, self.d_out, max_tokens, w_base_tiled.device)

    def __call__(self, x: torch.Tensor, seg_offsets: Sequence[int], y: Optional[torch.Tensor] = None) -> torch.Tensor:
        T = x.shape[0]
        if y is None:
            y = torch.empty((T, self.d_out), dtype=torch.bfloat16, device=x.device)
        seg = (ctypes.c_int32 * (self.E + 1))(*seg_offsets)
        _check(lib.mes_delta_linear(_ptr(self.w), self.desc, self.E, _ptr(x), T, seg, _ptr(y), _ptr(self.ws),
                                    self.ws.numel(), _stream(x.device)))
        return y


def mes_delta_linear(w_base_tiled, experts, x, seg_offsets, y=None, workspace=None):
    return DeltaLinear(w_base_tiled, experts, x.shape[0], workspace)(x, seg_offsets, y)


def mes_delta_linear_noalloc(w_base_tiled: torch.Tensor, experts: Sequence[PackedDelta], x: torch.Tensor,
                             seg_offsets: Sequence[int], y: torch.Tensor) -> torch.Tensor:
    """mes_delta_linear_noalloc: the scratch is the library's device-resident static array; y is the caller's."""
    E, T = len(experts), x.shape[0]
    desc = (mes_delta * E)(*[e.descriptor() for e in experts])
    seg = (ctypes.c_int32 * (E + 1))(*seg_offsets)
    _check(lib.mes_delta_linear_noalloc(_ptr(w_base_tiled), desc, E, _ptr(x), T, seg, _ptr(y), _stream(x.device)))
    return y


def mes_delta_linear_descriptors(w_base_tiled: torch.Tensor, desc, x: torch.Tensor, seg_offsets: Sequence[int],
                                 workspace: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """mes_delta_linear on a ready ctypes array of mes_delta (e.g. what ExpertPool.acquire returns)."""
    E, T, d_out = len(desc), x.shape[0], desc[0].d_out
    if y is None:
        y = torch.empty((T, d_out), dtype=torch.bfloat16, device=x.device)
    seg = (ctypes.c_int32 * (E + 1))(*seg_offsets)
    _check(lib.mes_delta_linear(_ptr(w_base_tiled), desc, E, _ptr(x), T, seg, _ptr(y), _ptr(workspace),
                                workspace.numel(), _stream(x.device)))
    return y


def mes_delta_linear_multi_descriptors(ws_tiled: Sequence[torch.Tensor], descs: Sequence, x: torch.Tensor,
                                       seg_offsets: Sequence[int], workspace: torch.Tensor,
                                       ys: Optional[Sequence[torch.Tensor]] = None):
    """mes_delta_linear_multi on ready ctypes arrays of mes_delta, one per layer (e.g. what a layer-spanning
    ExpertPool.acquire returns)."""
    n, E, T = len(descs), len(descs[0]), x.shape[0]
    if ys is None:
        ys = [torch.empty((T, d[0].d_out), dtype=torch.bfloat16, device=x.device) for d in descs]
    lin = (mes_linear * n)(*[mes_linear(ws_tiled[l].data_ptr(), descs[l], ys[l].data_ptr()) for l in range(n)])
    seg = (ctypes.c_int32 * (E + 1))(*seg_offsets)
    _check(lib.mes_delta_linear_multi(lin, n, E, _ptr(x), T, seg, _ptr(workspace), workspace.numel(), _stream(x.device)))
    return list(ys)


class DeltaLinearMulti:
    """Marshalled arguments of mes_delta_linear_multi: several layers that read the same activations and routing."""

    def __init__(self, layers: Sequence, max_tokens: int = 64, workspace: Optional[torch.Tensor] = None):
        """layers: sequence of (w_base_tiled, [PackedDelta per expert]).  workspace: a workspace of at
        least workspace_bytes(...) bytes to share between calls that are stream-ordered, or None to allocate one."""
        self.ws_tiled = [w for w, _ in layers]
        self.experts = [list(ex) for _, ex in layers]
        self.n = len(layers)
        self.E = len(self.experts[0])
        self.d_in = self.experts[0][0].d_in
        self.d_out = [ex[0].d_out for ex in self.experts]
        self.desc = [(mes_delta * self.E)(*[e.descriptor() for e in ex]) for ex in self.experts]
        dev = self.ws_tiled[0].device
        d = (ctypes.c_int32 * self.n)(*self.d_out)
        nbytes = max(lib.mes_linear_multi_workspace_bytes(self.d_in, d, self.n, max_tokens), 16)
        if workspace is not None:
            assert workspace.numel() >= nbytes
            self.ws = workspace
        else:
            self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    @staticmethod
    def workspace_bytes(d_in: int, d_outs: Sequence[int], max_tokens: int) -> int:
        d = (ctypes.c_int32 * len(d_outs))(*d_outs)
        return max(lib.mes_linear_multi_workspace_bytes(d_in, d, len(d_outs), max_tokens), 16)

    def __call__(self, x: torch.Tensor, seg_offsets: Sequence[int], ys: Optional[Sequence[torch.Tensor]] = None):
        T = x.shape[0]
        if ys is None:
            ys = [torch.empty((T, d), dtype=torch.bfloat16, device=x.device) for d in self.d_out]
        lin = (mes_linear * self.n)(*[mes_linear(self.ws_tiled[l].data_ptr(), self.desc[l], ys[l].data_ptr())
                                      for l in range(self.n)])
        seg = (ctypes.c_int32 * (self.E + 1))(*seg_offsets)
        _check(lib.mes_delta_linear_multi(lin, self.n, self.E, _ptr(x), T, seg, _ptr(self.ws), self.ws.numel(),
                                          _stream(x.device)))
        return list(ys)


class DeltaLinearGated:
    """Marshalled arguments of mes_delta_linear_gated: h = SiLU(gate layer) * (up layer), one pass, one output."""

    def __init__(self, w_gate_tiled, gate_experts, w_up_tiled, up_experts, max_tokens: int = 64,
                 workspace: Optional[torch.Tensor] = None):
        self.w_gate, self.w_up = w_gate_tiled, w_up_tiled
        self.gate, self.up = list(gate_experts), list(up_experts)
        self.E = len(self.gate)
        self.d_in, self.d_out = self.gate[0].d_in, self.gate[0].d_out
        self.gate_desc = (mes_delta * self.E)(*[e.descriptor() for e in self.gate])
        self.up_desc = (mes_delta * self.E)(*[e.descriptor() for e in self.up])
        nbytes = max(lib.mes_gated_workspace_bytes(self.d_in, self.d_out, max_tokens), 16)
        self.ws = workspace if workspace is not None else torch.empty(nbytes, dtype=torch.uint8, device=w_gate_tiled.device)
        assert self.ws.numel() >= nbytes

    def __call__(self, x: torch.Tensor, seg_offsets: Sequence[int], h: Optional[torch.Tensor] = None) -> torch.Tensor:
        T = x.shape[0]
        if h is None:
            h = torch.empty((T, self.d_out), dtype=torch.bfloat16, device=x.device)
        seg = (ctypes.c_int32 * (self.E + 1))(*seg_offsets)
        _check(lib.mes_delta_linear_gated(_ptr(self.w_gate), self.gate_desc, _ptr(self.w_up), self.up_desc, self.E, _ptr(x), T,
                                          seg, _ptr(h), _ptr(self.ws), self.ws.numel(), _stream(x.device)))
        return h


class ExpertPool:
    """On-demand swapping (mes_pool_* in mes.h): a device arena of `n_slots` slots and one pinned host blob per
    registered expert.  d_in, d_out, k: ints for a pool over one linear layer, or equally long sequences for a pool
    whose slots hold an expert's deltas of several layers (a miss is one copy either way)."""

    def __init__(self, d_in, d_out, k, bits: int, grid: int, n_slots: int, n_experts: int,
                 device="cuda:0", dry_run: bool = False):
        self.single = isinstance(d_in, int)
        as_list = lambda v: [int(v)] if isinstance(v, int) else [int(a) for a in v]
        self.d_in, self.d_out, self.k = as_list(d_in), as_list(d_out), as_list(k)
        self.n_linears = len(self.d_in)
        assert len(self.d_out) == self.n_linears and len(self.k) == self.n_linears
        self.bits, self.grid = bits, grid
        self.n_slots = n_slots
        arr = lambda v: (ctypes.c_int32 * self.n_linears)(*v)
        self.slot_bytes = lib.mes_pool_multi_slot_bytes(self.n_linears, arr(self.d_in), arr(self.d_out), arr(self.k), bits)
        if dry_run:
            self.arena, arena_ptr = None, 256          # any aligned non-null address: a dry-run pool never touches it
        else:
            self.arena = torch.empty(self.slot_bytes * n_slots, dtype=torch.uint8, device=device)
            arena_ptr = self.arena.data_ptr()
            self.copy_stream = torch.cuda.Stream(device=device)
        self.device = device
        self.dry_run = dry_run
        self.host = {}                                  # expert -> pinned host blob (kept alive here)
        h = ctypes.c_void_p()
        _check(lib.mes_pool_create_multi(self.n_linears, arr(self.d_in), arr(self.d_out), arr(self.k), bits, grid, n_slots,
                                         n_experts, arena_ptr, self.slot_bytes * n_slots, int(dry_run), ctypes.byref(h)))
        self.handle = h
        # where each linear's buffers sit inside a slot / blob
        self.offsets = []
        for l in range(self.n_linears):
            off = (ctypes.c_size_t * 4)()
            lib.mes_pool_slot_layout(self.d_in[l], self.d_out[l], self.k[l], bits, off)
            base = lib.mes_pool_linear_offset(self.handle, l)
            self.offsets.append([base + int(o) for o in off])

    def register(self, expert: int, packed) -> None:
        """packed: a PackedDelta (single-linear pool) or one per linear.  Builds the expert's blob in pinned host
        memory and registers it."""
        packed = [packed] if self.single and not isinstance(packed, (list, tuple)) else list(packed)
        assert len(packed) == self.n_linears
        blob = torch.zeros(self.slot_bytes, dtype=torch.uint8, pin_memory=True)
        for l, pk in enumerate(packed):
            for off, t in zip(self.offsets[l], (pk.codes, pk.step, pk.salient, pk.salient_idx)):
                if t is None or t.numel() == 0:
                    continue
                raw = t.contiguous().view(torch.uint8).reshape(-1)
                blob[off: off + raw.numel()].copy_(raw)
        if expert in self.host and not self.dry_run:
            # a copy out of the blob this one replaces may still be in flight
            self.copy_stream.synchronize()
        _check(lib.mes_pool_register_blob(self.handle, expert, blob.data_ptr()))
        self.host[expert] = blob

    def register_raw(self, expert: int, codes: int, step: int, salient: int, sidx: int) -> None:
        _check(lib.mes_pool_register(self.handle, expert, codes, step, salient, sidx))

    def _streams(self):
        if self.dry_run:
            return None, None
        return self.copy_stream.cuda_stream, _stream(torch.device(self.device))

    def acquire(self, experts: Sequence[int]):
        """Makes `experts` resident; returns the ctypes array of their descriptors (valid until the next acquire):
        [n] for a single-linear pool, else a list with one such array per linear."""
        n = len(experts)
        ids = (ctypes.c_int32 * n)(*experts)
        out = (mes_delta * (n * self.n_linears))()
        cs, ks = self._streams()
        _check(lib.mes_pool_acquire_multi(self.handle, ids, n, out, cs, ks))
        if self.single:
            return out
        size = ctypes.sizeof(mes_delta) * n
        return [(mes_delta * n).from_buffer(out, l * size) for l in range(self.n_linears)]   # views: `out` stays alive with them

    def prefetch(self, experts: Sequence[int]) -> int:
        """Starts loading the experts that are not resident into slots the latest acquire did not hand out; returns
        how many copies were started."""
        n = len(experts)
        ids = (ctypes.c_int32 * n)(*experts)
        loaded = ctypes.c_int(0)
        cs, _ = self._streams()
        _check(lib.mes_pool_prefetch(self.handle, ids, n, ctypes.byref(loaded), cs))
        return loaded.value

    def slot_of(self, expert: int) -> int:
        return lib.mes_pool_slot_of(self.handle, expert)

    def stats(self):
        h, m, b = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
        _check(lib.mes_pool_stats(self.handle, ctypes.byref(h), ctypes.byref(m), ctypes.byref(b)))
        return h.value, m.value, b.value

    def prefetched(self) -> int:
        return lib.mes_pool_prefetched(self.handle)

    def __del__(self):
        if getattr(self, "handle", None):
            lib.mes_pool_destroy(self.handle)
            self.handle = None


# ---------------------------------------------------------------------------------------- attention and its paged cache

# These calls take microseconds, and so do torch's friendlier forms of the questions below.
_BF16, _INT32 = torch.bfloat16, torch.int32
_raw_stream, _current = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device


def _call_on(index: int, entry, *args) -> None:
    """entry(*args, stream) on the current stream of device `index`, with that device current during the call."""
    if _current() == index:
        status = entry(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = entry(*args, _raw_stream(index))
    if status:
        _check(status)


def _rows(name: str, t: torch.Tensor, index: int, dtype: torch.dtype = _BF16):
    """Checks rows [T, heads, head_dim] of bf16 (or another type) on device `index` whose heads lie one behind the other: T, heads,
    head_dim, and how far rows are apart."""
    n, heads, dim = t.shape
    step, head, one = t.stride()
    assert t.dtype is dtype and t.get_device() == index and (one == 1 or dim == 1) and (head == dim or heads == 1), \
        f"{name}: {dtype} [T, heads, head_dim] on device {index}, the heads of a row one behind the other"
    return n, heads, dim, step if n > 1 else heads * dim


def _int32_on(name: str, t: torch.Tensor, index: int) -> None:
    assert t.dtype is _INT32 and t.get_device() == index and t.is_contiguous(), f"{name}: contiguous int32 on device {index}"


class KvCache:
    """A paged cache of keys and values for all layers of a model (mes_kv in mes.h): k and v are
    [n_layers, n_pages, n_kv_heads, page_tokens, head_dim], bf16, or float8_e4m3fn with k_scale and v_scale: one fp32 scale per layer and
    head (KV_E4M3), or exponents of blocks of 16 tokens, float8_e8m0fnu [n_layers, n_pages, n_kv_heads, page_tokens / 16]
    (KV_E4M3_BLOCKS), which mes_kv_append finds."""

    def __init__(self, n_layers: int, n_pages: int, page_tokens: int, n_kv_heads: int, head_dim: int, dtype: int = KV_BF16,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, device="cuda:0"):
        shape = (n_layers, n_pages, n_kv_heads, page_tokens, head_dim)
        if dtype == KV_E4M3_BLOCKS:
            assert k_scale is None and v_scale is None, "a cache of blocks finds its exponents itself"
            k_scale, v_scale = (torch.full((*shape[:3], page_tokens // KV_BLOCK), LEAST_EXPONENT, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu)
                                for _ in range(2))
        kind = torch.bfloat16 if dtype == KV_BF16 else torch.float8_e4m3fn
        self._set(*(torch.zeros(shape, dtype=kind if dtype == KV_BF16 else torch.uint8, device=device).view(kind) for _ in range(2)), k_scale, v_scale)

    @classmethod
    def over(cls, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        """A cache over tensors that are there already."""
        self = cls.__new__(cls)
        self._set(k, v, k_scale, v_scale)
        return self

    def _set(self, k, v, k_scale, v_scale):
        assert k.dim() == 5 and k.shape == v.shape and k.dtype == v.dtype and k.is_contiguous() and v.is_contiguous() and k.is_cuda and k.device == v.device
        assert k.dtype in (torch.bfloat16, torch.float8_e4m3fn), "a cache is bf16 or float8_e4m3fn"
        fp8 = k.dtype == torch.float8_e4m3fn
        blocks = fp8 and k_scale is not None and k_scale.dtype == torch.float8_e8m0fnu
        for t in (k_scale, v_scale):
            assert (t is not None) == fp8, "scales belong to an e4m3 cache"
            kind, shape = (torch.float8_e8m0fnu, (*k.shape[:3], k.shape[3] // KV_BLOCK)) if blocks else (torch.float32, (k.shape[0], k.shape[2]))
            assert t is None or (t.dtype == kind and t.shape == shape and t.is_contiguous() and t.device == k.device)
        self.k, self.v, self.k_scale, self.v_scale, self.device, self.index = k, v, k_scale, v_scale, k.device, k.get_device()
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = k.shape
        self.dtype = KV_E4M3_BLOCKS if blocks else KV_E4M3 if fp8 else KV_BF16
        self.desc = mes_kv(self.n_layers, self.n_pages, self.page_tokens, self.n_kv_heads, self.head_dim, self.dtype,
                           k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if fp8 else None, v_scale.data_ptr() if fp8 else None)
        self.ref = ctypes.byref(self.desc)


class SeqBatch:
    """The sequences of a call (mes_seqs in mes.h): kv_len int32 [n], page_table int32 [n, pages], q_offsets int32 [n + 1] or
    None (one row per sequence), all on the GPU; their contents may change between calls."""

    def __init__(self, kv_len: torch.Tensor, page_table: torch.Tensor, q_offsets: Optional[torch.Tensor] = None):
        self.index = kv_len.get_device()
        n = kv_len.shape[0]
        _int32_on("kv_len", kv_len, self.index)
        _int32_on("page_table", page_table, self.index)
        assert kv_len.is_cuda and kv_len.dim() == 1 and page_table.dim() == 2 and page_table.shape[0] == n
        if q_offsets is not None:
            _int32_on("q_offsets", q_offsets, self.index)
            assert q_offsets.shape == (n + 1,)
        self.kv_len, self.page_table, self.q_offsets, self.n = kv_len, page_table, q_offsets, n
        self.desc = mes_seqs(n, page_table.shape[1], None if q_offsets is None else q_offsets.data_ptr(), kv_len.data_ptr(), page_table.data_ptr())
        self.ref = ctypes.byref(self.desc)


def rotary_table(n_positions: int, head_dim: int, base: float = 10000.0, device="cuda:0") -> torch.Tensor:
    """Cosines and sines [n_positions, 2, head_dim / 2] for mes_kv_append; angles in fp64 (they pass what fp32 resolves)."""
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)
    return torch.stack([angle.cos(), angle.sin()], 1).to(device=device, dtype=torch.float32)


def mes_rotary_table(n_positions: int, dims: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, context: int = 0,
                     low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, device="cuda:0", out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Cosines and sines [n_positions, 2, dims / 2], fp32, made on the GPU (mes_rotary_table in mes.h).  scaling, for contexts `factor` times
    as long as trained at: None, "linear", "base", or "bands" (dimensions that turn `high` times or more over the trained `context` stay as
    they are, those that turn `low` times or fewer are stretched).  magnitude: multiplies all of it."""
    assert scaling in SCALINGS, f"scaling = {scaling!r}: None, 'linear', 'base' or 'bands'"
    if out is None:
        out = torch.empty((max(n_positions, 0), 2, max(dims, 0) // 2), dtype=torch.float32, device=device)
    assert out.is_cuda and out.dtype is torch.float32 and out.is_contiguous() and out.shape == (n_positions, 2, dims // 2)
    _call_on(out.get_device(), lib.mes_rotary_table, out.data_ptr(), n_positions, dims, base, SCALINGS[scaling], factor, context, low, high, magnitude)
    return out


class Angles:
    """Rotary angles (mes_angles in mes.h): table fp32 [n_positions, 2, dims / 2] as from mes_rotary_table or rotary_table, dims of them turned, where
    dimension i turns with i + dims / 2, or (interleaved) 2 i with 2 i + 1."""

    def __init__(self, table: torch.Tensor, interleaved: bool = False):
        assert table.is_cuda and table.dtype is torch.float32 and table.is_contiguous() and table.dim() == 3 and table.shape[1] == 2
        self.table, self.index, self.dims = table, table.get_device(), 2 * table.shape[2]
        self.desc = mes_angles(table.data_ptr(), table.shape[0], self.dims, ROTARY_PAIRS if interleaved else ROTARY_HALVES)
        self.ref = ctypes.byref(self.desc)


class _Turned(torch.autograd.Function):
    """mes_rotary with a graph behind it: the gradients of the rows are those of the turned rows, turned back."""

    @staticmethod
    def forward(ctx, angles, positions, transpose, *rows):
        ctx.angles, ctx.transpose = angles, transpose
        ctx.save_for_backward(positions, angles.table)       # neither may be written to until the gradients are there
        ctx.set_materialize_grads(False)
        return mes_rotary(angles, positions, *rows, transpose=transpose)

    @staticmethod
    def backward(ctx, *grads):
        positions, _ = ctx.saved_tensors
        grads = [g if need else None for g, need in zip(grads, ctx.needs_input_grad[3:])]
        there = [g.contiguous() for g in grads if g is not None]
        back = mes_rotary(ctx.angles, positions, *there, transpose=not ctx.transpose) if there else ()
        back = iter(back if len(there) == 2 else (back,))
        return (None, None, None, *(None if g is None else next(back) for g in grads))


def mes_rotary(angles: Angles, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               k_out: Optional[torch.Tensor] = None, transpose: bool = False):
    """Turns rows q [T, heads, d] and k [T, kv heads, d], bf16 or fp32, by the angles of positions int32 [T]; returns (q_out, k_out), or q_out
    where there is no k (q_out may be q, k_out k).  transpose: turns back, which takes gradients of turned rows to those of the rows.
    Rows whose position is outside the table (-1) are left as they are in outputs that are given, and 0 where these are allocated.
    Rows that require gradients: outputs that are allocated are part of the graph, and none can be given."""
    index, kind = q.get_device(), q.dtype
    if torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad)):
        assert q_out is None and k_out is None, "q_out, k_out: rows that require gradients are turned into outputs that are allocated"
        return _Turned.apply(angles, positions, transpose, *((q,) if k is None else (q, k)))
    assert kind in (_BF16, torch.float32) and q.is_cuda and angles.index == index, "rows are bf16 or fp32, on the angles' device"
    T, heads, dim, ld_q = _rows("q", q, index, kind)
    _int32_on("positions", positions, index)
    assert positions.shape == (T,), f"positions: int32 [{T}]"
    assert (k is None) <= (k_out is None) and (k is None or (q_out is None) == (k_out is None)), "give both of q_out and k_out or neither"
    kv_heads = ld_k = ld_ko = 0
    fresh = q_out is None
    if fresh:
        q_out, ld_qo = torch.empty((T, heads, dim), dtype=kind, device=q.device), heads * dim
    else:
        n, h, d, ld_qo = _rows("q_out", q_out, index, kind)
        assert (n, h, d) == (T, heads, dim)
    if k is not None:
        n, kv_heads, d, ld_k = _rows("k", k, index, kind)
        assert (n, d) == (T, dim), "k: as many rows as q"
        if fresh:
            k_out, ld_ko = torch.empty((T, kv_heads, dim), dtype=kind, device=q.device), kv_heads * dim
        else:
            n, h, d, ld_ko = _rows("k_out", k_out, index, kind)
            assert (n, h, d) == (T, kv_heads, dim)
    _call_on(index, lib.mes_rotary, angles.ref, positions.data_ptr(), q.data_ptr(), None if k is None else k.data_ptr(), T, heads, kv_heads, dim, ld_q, ld_k,
             0 if kind is _BF16 else 1, int(transpose), q_out.data_ptr(), ld_qo, None if k is None else k_out.data_ptr(), ld_ko, int(fresh))
    return q_out if k is None else (q_out, k_out)


def mes_kv_append(cache: KvCache, layer: int, batch: SeqBatch, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                  rotary=None, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Rotates the new rows' queries (returned; q_out may be q) and keys and puts keys and values into the cache's pages.  rotary: a table
    [n, 2, head_dim / 2] (rotary_table), Angles of any form, or None.  Rows without a position are left as they are in a q_out that is given, and 0
    where it is allocated."""
    index = cache.index
    T, kv_heads, dim, ld_k = _rows("k", k, index)
    rows_v = _rows("v", v, index)
    assert batch.index == index and rows_v[:3] == (T, kv_heads, dim) == (T, cache.n_kv_heads, cache.head_dim), "k, v: [T, n_kv_heads, head_dim] of the cache"
    heads = ld_q = ld_o = n_pos = 0
    rot = src = dst = None
    fresh, turned = q is not None and q_out is None, type(rotary) is Angles
    if turned:
        assert rotary.index == index, f"angles on device {index}"
    elif rotary is not None:
        assert rotary.dtype is torch.float32 and rotary.is_contiguous() and rotary.get_device() == index and rotary.shape[1:] == (2, dim // 2)
        n_pos, rot = rotary.shape[0], rotary.data_ptr()
    if q is not None:
        n, heads, d, ld_q = _rows("q", q, index)
        assert n == T and d == dim
        if fresh:
            q_out, ld_o = torch.empty_like(q, memory_format=torch.contiguous_format), heads * dim
        else:
            n, h, d, ld_o = _rows("q_out", q_out, index)
            assert (n, h, d) == (T, heads, dim)
        src, dst = q.data_ptr(), q_out.data_ptr()
    if turned:
        _call_on(index, lib.mes_kv_append_angles, cache.ref, layer, batch.ref, src, k.data_ptr(), v.data_ptr(), T, heads, ld_q, ld_k, rows_v[3], rotary.ref,
                 dst, ld_o, fresh)
    else:
        _call_on(index, lib.mes_kv_append_fresh if fresh else lib.mes_kv_append, cache.ref, layer, batch.ref, src, k.data_ptr(), v.data_ptr(), T, heads, ld_q,
                 ld_k, rows_v[3], rot, n_pos, dst, ld_o)
    return q_out if q is not None else None


def mes_kv_read(cache: KvCache, layer: int, batch: SeqBatch, T: int, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """Reads the tokens of the batch's T rows (the last tokens of their sequences, as in mes_kv_append) back: k, v bf16 [T, kv heads, head_dim].  Given
    one of k_out and v_out, only that is read.  Rows of a sequence whose token is absent are 0; rows behind the last
    sequence are left as they are in outputs that are given, and 0 where these are allocated."""
    index = cache.index
    assert batch.index == index
    fresh, heads, dim = k_out is None and v_out is None, cache.n_kv_heads, cache.head_dim
    ld = [heads * dim] * 2
    if fresh:
        k_out, v_out = torch.empty((2, max(T, 0), heads, dim), dtype=_BF16, device=cache.device)
    else:
        for i, t in enumerate((k_out, v_out)):
            if t is not None:
                *shape, ld[i] = _rows("k_out / v_out", t, index)
                assert shape == [T, heads, dim], "k_out, v_out: [T, n_kv_heads, head_dim] of the cache"
    _call_on(index, lib.mes_kv_read, cache.ref, layer, batch.ref, T, None if k_out is None else k_out.data_ptr(), None if v_out is None else v_out.data_ptr(),
             *ld, int(fresh))
    return k_out, v_out


def _scratch(workspace: Optional[torch.Tensor], index: int):
    if workspace is None:
        return None, 0
    assert workspace.get_device() == index and workspace.dtype is torch.uint8 and workspace.is_contiguous()
    return workspace.data_ptr(), workspace.numel()


def prompt_workspace(T: int, n_seqs: int, n_heads: int, n_kv_heads: int, head_dim: int, device) -> torch.Tensor:
    """Allocates a workspace of mes_attn_prompt / mes_attn_extend (scratch: its contents do not matter)."""
    return torch.empty(lib.mes_attn_prompt_workspace_bytes(T, n_seqs, n_heads, n_kv_heads, head_dim), dtype=torch.uint8, device=device)


def mes_attn_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seq_offsets: torch.Tensor, out: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal attention over packed prompts: q [T, heads, d], k and v [T, kv heads, d] (views of one buffer are fine),
    seq_offsets int32 [n + 1] on the GPU.  Returns [T, heads, d]; rows behind the last sequence are left as they are.
    workspace: one to share between stream-ordered calls (prompt_workspace), or None to allocate one."""
    index = q.get_device()
    T, heads, dim, ld_q = _rows("q", q, index)
    n, kv_heads, d, ld_k = _rows("k", k, index)
    rows_v = _rows("v", v, index)
    assert rows_v[:3] == (n, kv_heads, d) == (T, kv_heads, dim) and q.is_cuda, "k, v: [T, kv heads, head_dim], as many rows as q"
    _int32_on("seq_offsets", seq_offsets, index)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    rows_o = _rows("out", out, index)
    assert rows_o[:3] == (T, heads, dim)
    n = seq_offsets.shape[0] - 1
    if workspace is None and T > SHORT_PROMPT:
        workspace = prompt_workspace(T, n, heads, kv_heads, dim, q.device)
    _call_on(index, lib.mes_attn_prompt, q.data_ptr(), k.data_ptr(), v.data_ptr(), T, n, seq_offsets.data_ptr(), heads, kv_heads, dim, ld_q, ld_k, rows_v[3],
             dim ** -0.5 if scale is None else scale, out.data_ptr(), rows_o[3], *_scratch(workspace, index))
    return out


def mes_attn_extend(cache: KvCache, layer: int, batch: SeqBatch, q: torch.Tensor, out: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal attention of the batch's new rows (its last tokens, already appended) over the cache.  workspace: as for
    mes_attn_prompt."""
    index = cache.index
    T, heads, dim, ld_q = _rows("q", q, index)
    assert batch.index == index and dim == cache.head_dim
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    rows_o = _rows("out", out, index)
    assert rows_o[:3] == (T, heads, dim)
    if workspace is None and batch.desc.table_pages * cache.page_tokens > SHORT_PROMPT:
        workspace = prompt_workspace(T, batch.n, heads, cache.n_kv_heads, dim, cache.device)
    _call_on(index, lib.mes_attn_extend, cache.ref, layer, batch.ref, q.data_ptr(), T, heads, ld_q, dim ** -0.5 if scale is None else scale,
             out.data_ptr(), rows_o[3], *_scratch(workspace, index))
    return out


class AttnDecode:
    """mes_attn_decode with its workspace, for up to max_seqs sequences; all layers of a model can share one, and calls follow one another
    on one stream (or wait for each other)."""

    def __init__(self, cache: KvCache, n_heads: int, max_seqs: int = 64, workspace: Optional[torch.Tensor] = None):
        self.cache, self.n_heads = cache, n_heads
        assert 0 <= max_seqs <= MAX_SEQS, f"max_seqs = {max_seqs} outside [0, {MAX_SEQS}]"
        n = lib.mes_attn_decode_workspace_bytes(max(max_seqs, 1), n_heads, cache.n_kv_heads, cache.head_dim)
        assert n, f"n_heads = {n_heads} must be 1 to 64 times the cache's {cache.n_kv_heads}, head_dim 64 or 128 (got {cache.head_dim})"
        self.ws = workspace if workspace is not None else torch.empty(n, dtype=torch.uint8, device=cache.device)
        self.scratch = _scratch(self.ws, cache.index)

    def __call__(self, layer: int, batch: SeqBatch, q: torch.Tensor, seg_offsets: Optional[Sequence[int]] = None,
                 prefix_len: Optional[Sequence[int]] = None, out: Optional[torch.Tensor] = None, scale: Optional[float] = None) -> torch.Tensor:
        """q [n, heads, d], one row per sequence.  seg_offsets [E + 1] and prefix_len [E] (host): rows are sorted by expert and
        the sequences of expert e share their first prefix_len[e] tokens, which are then read once."""
        cache, index = self.cache, self.cache.index
        n, heads, dim, ld_q = _rows("q", q, index)
        assert batch.index == index and n == batch.n and heads == self.n_heads and dim == cache.head_dim
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        rows_o = _rows("out", out, index)
        assert rows_o[:3] == (n, heads, dim)
        E, seg, pre = 0, None, None
        if seg_offsets is not None:
            E = len(prefix_len)
            assert len(seg_offsets) == E + 1
            seg, pre = (ctypes.c_int32 * (E + 1))(*seg_offsets), (ctypes.c_int32 * E)(*prefix_len)
        _call_on(index, lib.mes_attn_decode, cache.ref, layer, batch.ref, q.data_ptr(), heads, ld_q, E, seg, pre,
                 dim ** -0.5 if scale is None else scale, out.data_ptr(), rows_o[3], *self.scratch)
        return out


def mes_kv_copy_pages(cache: KvCache, src: Sequence[int], dst: Sequence[int]) -> None:
    """Copies page src[i] to page dst[i] in all layers of keys and values (what PagePool.grow and .compact ask for)."""
    n = len(src)
    assert len(dst) == n
    pages = ctypes.c_int32 * n
    _call_on(cache.index, lib.mes_kv_copy_pages, cache.ref, pages(*src), pages(*dst), n)


class PagePool:
    """Which pages of a cache hold which sequence (mes_pages_* in mes.h; host bookkeeping only)."""

    def __init__(self, n_pages: int, page_tokens: int, max_seqs: int, max_seq_pages: Optional[int] = None):
        self.n_pages, self.page_tokens, self.max_seqs = n_pages, page_tokens, max_seqs
        self.max_seq_pages = n_pages if max_seq_pages is None else max_seq_pages
        h = ctypes.c_void_p()
        _check(lib.mes_pages_create(n_pages, page_tokens, max_seqs, self.max_seq_pages, ctypes.byref(h)))
        self.handle = h

    def grow(self, seqs: Sequence[int], n_tokens: Sequence[int]):
        """More tokens for each of the sequences; returns (src, dst): pages to copy before the tokens are appended."""
        n = len(seqs)
        assert len(n_tokens) == n
        arr, count = ctypes.c_int32 * max(n, 1), ctypes.c_int(0)
        src, dst = arr(), arr()
        _check(lib.mes_pages_grow(self.handle, arr(*seqs), arr(*n_tokens), n, src, dst, ctypes.byref(count)))
        return src[: count.value], dst[: count.value]

    def fork(self, parent: int, child: int, n_tokens: Optional[int] = None) -> None:
        _check(lib.mes_pages_fork(self.handle, parent, child, self.length(parent) if n_tokens is None else n_tokens))

    def free(self, seq: int) -> None:
        _check(lib.mes_pages_free(self.handle, seq))

    def compact(self):
        """Moves the pages in use to the lowest ids; returns (src, dst) to copy.  Tables taken before are out of date."""
        arr, count = ctypes.c_int32 * max(self.n_pages // 2, 1), ctypes.c_int(0)
        src, dst = arr(), arr()
        _check(lib.mes_pages_compact(self.handle, src, dst, ctypes.byref(count)))
        return src[: count.value], dst[: count.value]

    def table(self, seqs: Sequence[int], table_pages: Optional[int] = None):
        """Host tensors (page_table [n, table_pages], kv_len [n]) of the sequences."""
        n = len(seqs)
        table = torch.empty((n, self.max_seq_pages if table_pages is None else table_pages), dtype=torch.int32)
        length = torch.empty(n, dtype=torch.int32)
        _check(lib.mes_pages_table(self.handle, (ctypes.c_int32 * max(n, 1))(*seqs), n, table.data_ptr() or None, table.shape[1], length.data_ptr() or None))
        return table, length

    def length(self, seq: int) -> int:
        return lib.mes_pages_length(self.handle, seq)

    def unused(self) -> int:
        return lib.mes_pages_unused(self.handle)

    def __del__(self):
        if getattr(self, "handle", None):
            lib.mes_pages_destroy(self.handle)
            self.handle = None


class KernelTimer:
    """HIP events recorded by the library around its dominant kernel (mes_time_next_call in mes_bench.h): `n` pairs,
    so that a whole sequence of calls can be timed without a synchronisation in between."""

    def __init__(self, n: int = 1):
        self.hip = ctypes.CDLL("libamdhip64.so")
        self.hip.hipEventCreate.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
        self.hip.hipEventSynchronize.argtypes = [ctypes.c_void_p]
        self.hip.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_void_p, ctypes.c_void_p]
        self.pairs = []
        for _ in range(n):
            pair = (ctypes.c_void_p(), ctypes.c_void_p())
            for ev in pair:
                if self.hip.hipEventCreate(ctypes.byref(ev)) != 0:
                    raise RuntimeError("hipEventCreate failed")
            self.pairs.append(pair)

    def arm(self, i: int = 0) -> None:
        """The next timed library call of this thread records pair i."""
        _check(lib.mes_time_next_call(self.pairs[i][0], self.pairs[i][1]))

    def elapsed_us(self, i: int = 0) -> float:
        start, stop = self.pairs[i]
        if self.hip.hipEventSynchronize(stop) != 0:
            raise RuntimeError("hipEventSynchronize failed")
        ms = ctypes.c_float()
        if self.hip.hipEventElapsedTime(ctypes.byref(ms), start, stop) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return ms.value * 1e3
