"""Thin ctypes binding over libspecdec.so (argument marshalling only).

Every function named ``specdec_*`` here calls the C entry point of the same
name; torch tensors are passed as device pointers and torch only provides
device memory and streams.  The classes bundle the buffers a caller owns
(weights, workspace, KV storage) with their handles.

The library must be built (``paper_2608_10362_amd.build.build()``); loading
fails loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Dict, Optional

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspecdec.so")

SPECDEC_F32, SPECDEC_BF16, SPECDEC_FP8 = 0, 1, 2
ROLE_TARGET, ROLE_DRAFT = 0, 1
INPUT_PROBS, INPUT_LOGITS = 0, 1
PURPOSE_DRAFT, PURPOSE_ACCEPT, PURPOSE_RESAMPLE = 0, 1, 2

STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported shape", -3: "KV capacity exceeded",
          -4: "non-finite probability or logit", -5: "HIP runtime error", -6: "unsupported request",
          -7: "token id out of range",
          -8: "request needs more scratch than the static no-allocation buffer holds",
          -9: "a kernel's bounded wait for other blocks ran out"}


# Size of the static scratch of specdec_accept_noalloc (SPECDEC_ACCEPT_NOALLOC_SCRATCH_BYTES).
ACCEPT_NOALLOC_SCRATCH_BYTES = 2 << 20


class SpecdecError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {STATUS.get(status, status)} ({status})")
        self.status = status


class ModelDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float), ("rope_base", ctypes.c_float),
                ("dtype", ctypes.c_int32)]


_PP = ctypes.POINTER(ctypes.c_void_p)


class Weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("lm_head", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("attn_norm", _PP), ("wq", _PP), ("wk", _PP), ("wv", _PP), ("wo", _PP), ("ffn_norm", _PP),
                ("w_gate", _PP), ("w_up", _PP), ("w_down", _PP)]


class KV(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("state", ctypes.c_void_p), ("batch", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("len_upper", ctypes.c_int64),
                ("window", ctypes.c_int32)]


class Sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("gain_dtype", ctypes.c_int32), ("q_gain", ctypes.c_void_p), ("k_gain", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("freq", ctypes.c_double * 64)]


_lib = None

_SIGS = {
    "specdec_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(ModelDesc), ctypes.c_int32, ctypes.c_int32]),
    "specdec_packed_bytes": (ctypes.c_size_t, [ctypes.POINTER(ModelDesc), ctypes.c_int32]),
    "specdec_packed_bytes_fmt": (ctypes.c_size_t, [ctypes.POINTER(ModelDesc), ctypes.c_int32, ctypes.c_int32]),
    "specdec_pack_weights_fmt": (ctypes.c_int, [ctypes.POINTER(ModelDesc), ctypes.POINTER(Weights), ctypes.c_int32,
                                                ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "specdec_model_create_fmt": (ctypes.c_int, [ctypes.POINTER(ModelDesc), ctypes.POINTER(Weights), ctypes.c_int32,
                                                ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32,
                                                ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t,
                                                ctypes.POINTER(ctypes.c_void_p)]),
    "specdec_pack_weights": (ctypes.c_int, [ctypes.POINTER(ModelDesc), ctypes.POINTER(Weights), ctypes.c_int32,
                                            ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "specdec_model_create": (ctypes.c_int, [ctypes.POINTER(ModelDesc), ctypes.POINTER(Weights), ctypes.c_int32,
                                            ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int32,
                                            ctypes.c_void_p, ctypes.c_size_t, ctypes.POINTER(ctypes.c_void_p)]),
    "specdec_model_destroy": (None, [ctypes.c_void_p]),
    "specdec_kv_bytes": (ctypes.c_size_t, [ctypes.POINTER(ModelDesc), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "specdec_kv_state_count": (ctypes.c_int32, [ctypes.c_int32]),
    "specdec_kv_init": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                       ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_write_context": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                                ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_read_context": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                               ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_set_state": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                            ctypes.c_void_p]),
    "specdec_kv_read_state": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_prefill": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_void_p,
                                       ctypes.c_void_p]),
    "specdec_draft_step": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32,
                                          ctypes.c_float, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                          ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_verify": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_void_p,
                                      ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_accept": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                      ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_size_t, ctypes.c_void_p]),
    "specdec_accept_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "specdec_accept_noalloc": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                              ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_int32, ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint64,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_void_p]),
    "specdec_packed_range": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                            ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]),
    "specdec_event_create": (ctypes.c_int, [ctypes.POINTER(ctypes.c_void_p)]),
    "specdec_event_destroy": (ctypes.c_int, [ctypes.c_void_p]),
    "specdec_load_async": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                          ctypes.c_void_p]),
    "specdec_stream_wait_event": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_event_query": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)]),
    "specdec_kv_commit": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_step_word": (ctypes.c_void_p, [ctypes.POINTER(KV)]),
    "specdec_sample": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64,
                                      ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int32,
                                      ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_bytes_fp8": (ctypes.c_size_t, [ctypes.POINTER(ModelDesc), ctypes.c_int32, ctypes.c_int32,
                                               ctypes.c_int32, ctypes.c_int32]),
    "specdec_kv_init_fp8": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.POINTER(ModelDesc), ctypes.c_int32,
                                           ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_append": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_kv_advance": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_void_p]),
    "specdec_attention_shared_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(KV), ctypes.POINTER(KV),
                                                                   ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "specdec_attention_shared": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.POINTER(KV),
                                                ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                ctypes.c_void_p]),
    "specdec_rope_init": (ctypes.c_int, [ctypes.POINTER(RopeDesc), ctypes.c_int32, ctypes.c_int32, ctypes.c_double,
                                         ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                         ctypes.c_float]),
    "specdec_rope_apply": (ctypes.c_int, [ctypes.POINTER(RopeDesc), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                          ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64,
                                          ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                          ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                          ctypes.c_int64, ctypes.c_void_p]),
    "specdec_rope_append": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.POINTER(RopeDesc),
                                           ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                           ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_attention_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32]),
    "specdec_attention": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                         ctypes.c_void_p]),
    "specdec_sample_logits_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "specdec_sample_logits": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                             ctypes.c_int64, ctypes.POINTER(Sampling), ctypes.c_void_p,
                                             ctypes.c_uint64, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                             ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                             ctypes.c_void_p]),
    "specdec_draw_u32": (ctypes.c_int, [ctypes.c_int32, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_device_status": (ctypes.c_int, [ctypes.POINTER(KV), ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "specdec_last_hip_error": (ctypes.c_char_p, []),
    "specdec_stream_read": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_timing_enable": (ctypes.c_int, [ctypes.c_int32]),
    "specdec_timing_read": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]),
    "specdec_time_kernel": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_void_p]),
}

KERNEL_KINDS = ("embed", "qkv", "rope_append", "attention", "o_proj", "gate_up", "down", "lm_head", "draft_finish",
                "accept", "commit")


def lib() -> ctypes.CDLL:
    """Load libspecdec.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2608_10362_amd.build.build()")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(l, name)
            f.restype = res
            f.argtypes = args
        _lib = l
    return _lib


def _check(status: int, what: str):
    if status != 0:
        if status == -5:  # name the HIP error behind it
            what = f"{what} [{lib().specdec_last_hip_error().decode()}]"
        raise SpecdecError(status, what)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t, name: str, dtype=None, numel: int = 0, optional: bool = False):
    """Check that a tensor argument is a contiguous device tensor of the right type and size."""
    import torch
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name}: missing")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.numel() < numel:
        raise ValueError(f"{name}: needs at least {numel} elements, has {t.numel()}")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    import torch
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    # the same handle without a Stream object: 0.2 us in place of 2.8 us a call
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _memory_of(stream):
    """Context in which a call launched on `stream` allocates: what is allocated for the
    current stream goes, once dropped, to that stream's next allocation, which
    does not wait for `stream`."""
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _after_current(stream):
    """`stream` waits for the current stream, on which a constructor has just allocated
    (and zeroed) what it now sets up on `stream`."""
    import torch
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())


def make_desc(shape) -> ModelDesc:
    return ModelDesc(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.head_dim, shape.ffn_dim,
                     shape.vocab, shape.rms_eps, shape.rope_base,
                     SPECDEC_BF16 if shape.dtype == "bf16" else SPECDEC_F32)


def workspace_bytes(shape, max_rows: int, max_ctx: int) -> int:
    d = make_desc(shape)
    return lib().specdec_workspace_bytes(ctypes.byref(d), max_rows, max_ctx)


def kv_bytes(shape, n_layers: int, batch: int, capacity: int) -> int:
    d = make_desc(shape)
    return lib().specdec_kv_bytes(ctypes.byref(d), n_layers, batch, capacity)


# ---------------------------------------------------------------- device weights
def _to_device(arr, dtype: str, device):
    import torch
    if isinstance(arr, torch.Tensor):
        return arr.to(device).contiguous()
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).view(torch.bfloat16).to(device)
    return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(device)


class DeviceWeights:
    """Device copies of a model's weights (from synth's numpy dict, or torch tensors).

    For bf16 models the matrices are packed once (specdec_pack_weights) into
    ``self.packed``; the row-major matrices are then released unless
    ``keep_rowmajor`` is set (the embedding and RMSNorm gains stay).
    """

    KEYS = ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")
    MATS = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")

    FORMATS = {"bf16": 0, "int4": 1}  # SPECDEC_WEIGHTS_*

    def __init__(self, shape, weights: Dict, device="cuda", keep_rowmajor: bool = False, stream=None,
                 weight_format: str = "bf16"):
        """``weight_format`` (bf16 models): "bf16", or "int4" for the INT4 image
        (layer matrices quantized on the device, see specdec_pack_weights_fmt)."""
        import torch
        if weight_format not in self.FORMATS or (weight_format != "bf16" and shape.dtype != "bf16"):
            raise ValueError(f"weight format {weight_format!r} for a {shape.dtype} model")
        self.weight_format = weight_format
        self.shape = shape
        self.t = {k: _to_device(weights[k], shape.dtype, device) for k in ("embed", "lm_head", "final_norm")}
        self.layers = [{k: _to_device(L[k], shape.dtype, device) for k in self.KEYS} for L in weights["layers"]]
        self.packed = None
        if shape.dtype == "bf16":
            desc = make_desc(shape.with_layers(self.n_layers))
            fmt = self.FORMATS[weight_format]
            nbytes = lib().specdec_packed_bytes_fmt(ctypes.byref(desc), self.n_layers, fmt)
            if nbytes == 0:
                raise SpecdecError(-2, "specdec_packed_bytes_fmt")
            self.packed = torch.empty(nbytes, dtype=torch.uint8, device=self.t["embed"].device)
            w, keep = self.c_struct(self.n_layers)
            _after_current(stream)
            _check(lib().specdec_pack_weights_fmt(ctypes.byref(desc), ctypes.byref(w), self.n_layers, fmt,
                                                  self.packed.data_ptr(), nbytes, _stream(stream)),
                   "specdec_pack_weights_fmt")
            torch.cuda.current_stream().synchronize() if stream is None else stream.synchronize()
            if not keep_rowmajor:
                self.t["lm_head"] = None
                for L in self.layers:
                    for k in self.MATS:
                        L[k] = None

    @property
    def n_layers(self):
        return len(self.layers)

    def c_struct(self, n_layers: int):
        arrays = {}
        for k in self.KEYS:
            arr = (ctypes.c_void_p * n_layers)(*[_ptr(self.layers[l][k]) for l in range(n_layers)])
            arrays[k] = arr
        w = Weights(self.t["embed"].data_ptr(), _ptr(self.t["lm_head"]), self.t["final_norm"].data_ptr(),
                    *[ctypes.cast(arrays[k], _PP) for k in self.KEYS])
        return w, arrays


class Model:
    """A model handle (target, or a draft = layer prefix) with its own workspace."""

    def __init__(self, dw: DeviceWeights, n_layers: int, max_rows: int, max_ctx: int, packed=None):
        """``packed``: a device image to run from instead of ``dw.packed`` (a
        draft slot, see DraftSlot); it must hold at least ``n_layers`` layers."""
        import torch
        self.dw = dw
        self.shape = dw.shape
        self.n_layers = n_layers
        self.max_rows = max_rows
        self.desc = make_desc(dw.shape.with_layers(dw.n_layers))
        nbytes = lib().specdec_workspace_bytes(ctypes.byref(self.desc), max_rows, max_ctx)
        if nbytes == 0:
            raise SpecdecError(-2, "specdec_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dw.t["embed"].device)
        w, self._arrays = dw.c_struct(n_layers)
        h = ctypes.c_void_p()
        pk = dw.packed if packed is None else packed
        if packed is not None:
            _dev(packed, "packed", torch.uint8, 1)
        self._packed = pk  # (kept alive with the handle)
        _check(lib().specdec_model_create_fmt(ctypes.byref(self.desc), ctypes.byref(w), n_layers,
                                              DeviceWeights.FORMATS[dw.weight_format], _ptr(pk),
                                              0 if pk is None else pk.numel(), max_rows, max_ctx,
                                              self.workspace.data_ptr(), nbytes, ctypes.byref(h)),
               "specdec_model_create_fmt")
        self.handle = h

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.specdec_model_destroy(self.handle)
            self.handle = None


class KVCache:
    """KV storage + sequence state of one model instance."""

    def __init__(self, model: Model, batch: int, capacity: int, stream=None):
        import torch
        self.model = model
        dev = model.workspace.device
        nbytes = lib().specdec_kv_bytes(ctypes.byref(model.desc), model.n_layers, batch, capacity)
        self.data = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        self.state = torch.zeros(lib().specdec_kv_state_count(batch), dtype=torch.int32, device=dev)
        self.kv = KV()
        _after_current(stream)
        _check(lib().specdec_kv_init(ctypes.byref(self.kv), model.handle, batch, capacity, self.data.data_ptr(),
                                     nbytes, self.state.data_ptr(), _stream(stream)), "specdec_kv_init")

    @property
    def batch(self):
        return self.kv.batch

    def storage_dtype(self):
        """Type of the K and V rows that go in and out (FP8 caches: bf16)."""
        import torch
        return torch.float32 if self.kv.dtype == SPECDEC_F32 else torch.bfloat16

    def write_context(self, layer: int, b: int, pos0: int, k, v, stream=None):
        n = k.shape[0]
        _dev(k, "k", self.storage_dtype(), n * self.kv.n_kv_heads * self.kv.head_dim)
        _dev(v, "v", self.storage_dtype(), n * self.kv.n_kv_heads * self.kv.head_dim)
        _check(lib().specdec_kv_write_context(ctypes.byref(self.kv), layer, b, pos0, k.shape[0], k.data_ptr(),
                                              v.data_ptr(), _stream(stream)), "specdec_kv_write_context")

    def read_context(self, layer: int, b: int, pos0: int, n: int, stream=None):
        """The rows as new tensors, valid once `stream` has run the copy; they may be
        dropped while the stream that was current at the call still reads them."""
        import torch
        shp = (n, self.kv.n_kv_heads, self.kv.head_dim)
        with _memory_of(stream):
            k = torch.empty(shp, dtype=self.storage_dtype(), device=self.data.device)
            v = torch.empty_like(k)
        if stream is not None:
            for t in (k, v):
                t.record_stream(torch.cuda.current_stream())
        _check(lib().specdec_kv_read_context(ctypes.byref(self.kv), layer, b, pos0, n, k.data_ptr(), v.data_ptr(),
                                             _stream(stream)), "specdec_kv_read_context")
        return k, v

    def set_state(self, length, pending, n_pending, stream=None):
        L = np.ascontiguousarray(length, dtype=np.int32)
        P = np.ascontiguousarray(pending, dtype=np.int32).reshape(-1)
        N = np.ascontiguousarray(n_pending, dtype=np.int32)
        _check(lib().specdec_kv_set_state(ctypes.byref(self.kv), L.ctypes.data, P.ctypes.data, N.ctypes.data,
                                          _stream(stream)), "specdec_kv_set_state")

    def read_state(self, stream=None):
        B = self.batch
        L = np.zeros(B, np.int32)
        P = np.zeros(2 * B, np.int32)
        N = np.zeros(B, np.int32)
        S = np.zeros(1, np.int32)
        _check(lib().specdec_kv_read_state(ctypes.byref(self.kv), L.ctypes.data, P.ctypes.data, N.ctypes.data,
                                           S.ctypes.data, _stream(stream)), "specdec_kv_read_state")
        return {"len": L, "pending": P.reshape(B, 2), "n_pending": N, "status": int(S[0])}

    def step_word(self) -> int:
        """Device address of the commit counter (the step_dev argument)."""
        return int(lib().specdec_kv_step_word(ctypes.byref(self.kv)))

    def read_step(self) -> int:
        """The commit counter's value (synchronizes the current stream)."""
        B = self.batch
        return int(self.state[4 * B + 2:4 * B + 4].cpu().numpy().view(np.uint64)[0])


def default_window(max_rows: int, batch: int, capacity: int) -> int:
    """The window of an Fp8KVCache for a handle of ``max_rows`` rows (0: none): what a
    prompt's chunk of these rows needs, at most a quarter of the capacity, at least 128.

    A prompt runs in chunks of window - 64 tokens per sequence, so a wide ring makes prefill
    faster, and is most of the cache where contexts are short.  Past 1024 rows a pass it
    brings nothing: 4096 tokens, 7B-like, four layers, 11.4 ms at a window of 2112 (as
    over a bf16 cache), 11.3 at 1088, 12.3 at 576, 20 at 256, 30 at 128."""
    need = (min(max_rows, 1024) // max(batch, 1) + 64 + 63) // 64 * 64
    return max(128, min(need, capacity // 4 // 64 * 64))


class Fp8KVCache(KVCache):
    """An 8-bit cache (see specdec_kv_init_fp8): takes the place of a KVCache of
    a bf16 model in every call, or serves a caller's own model through
    specdec_kv_append, specdec_attention and specdec_kv_advance.  ``of``: the
    Model that uses it, or a model shape (then ``n_layers`` of it).  ``window``:
    positions of the bf16 ring, default_window's if not given; a verify pass or an append of
    n rows a sequence needs n + 63.  Bytes, as a share of a bf16 cache's: 0.5 and a
    little, and window / capacity."""

    def __init__(self, of, batch: int, capacity: int, window: Optional[int] = None, n_layers: Optional[int] = None,
                 device="cuda", stream=None):
        import torch
        self.model = of if isinstance(of, Model) else None
        if self.model is not None:
            desc, device = of.desc, of.workspace.device
            n_layers = of.n_layers if n_layers is None else n_layers
        else:
            desc = make_desc(of)
            n_layers = of.n_layers if n_layers is None else n_layers
        if window is None:
            window = default_window(0 if self.model is None else of.max_rows, batch, capacity)
        nbytes = lib().specdec_kv_bytes_fp8(ctypes.byref(desc), n_layers, batch, capacity, window)
        if nbytes == 0:
            raise SpecdecError(-2, "specdec_kv_bytes_fp8")
        self.data = torch.empty(nbytes, dtype=torch.uint8, device=device)
        _on_current(self.data, "device", torch.uint8)
        self.state = torch.zeros(lib().specdec_kv_state_count(batch), dtype=torch.int32, device=device)
        self.kv = KV()
        _after_current(stream)
        _check(lib().specdec_kv_init_fp8(ctypes.byref(self.kv), ctypes.byref(desc), n_layers, batch, capacity, window,
                                         self.data.data_ptr(), nbytes, self.state.data_ptr(), _stream(stream)),
               "specdec_kv_init_fp8")


# ---------------------------------------------------------------- draft reload
def packed_range(shape, first_layer: int, n_layers: int):
    """(offset, bytes) of layers [first_layer, first_layer + n_layers) in the packed image."""
    d = make_desc(shape)
    off, nb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().specdec_packed_range(ctypes.byref(d), first_layer, n_layers, ctypes.byref(off), ctypes.byref(nb)),
           "specdec_packed_range")
    return off.value, nb.value


class Event:
    """A completion event owned by the library (see specdec_event_create)."""

    def __init__(self):
        h = ctypes.c_void_p()
        _check(lib().specdec_event_create(ctypes.byref(h)), "specdec_event_create")
        self.handle = h

    def query(self) -> bool:
        done = ctypes.c_int32(0)
        _check(lib().specdec_event_query(self.handle, ctypes.byref(done)), "specdec_event_query")
        return bool(done.value)

    def wait(self, stream=None):
        """Make `stream` (default: the current one) wait for the event."""
        _check(lib().specdec_stream_wait_event(_stream(stream), self.handle), "specdec_stream_wait_event")

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.specdec_event_destroy(self.handle)
            self.handle = None


class DraftSlot:
    """One resident draft slot: a device buffer in the packed-image format for
    drafts of up to ``max_layers`` layers (drafts are layer prefixes of the
    target, so their images are prefixes of its image).  The backing storage
    is a pinned host copy of that image prefix.  The shared LM head is copied
    into the slot once; ``load_async`` then re-sends only the layers of the
    draft being made resident, on ``copy_stream``, and ``event`` completes when
    they have landed."""

    def __init__(self, dw: DeviceWeights, max_layers: int):
        import torch
        if dw.packed is None:
            raise ValueError("draft slots hold packed (bf16) images")
        self.shape = dw.shape.with_layers(dw.n_layers)
        self.max_layers = max_layers
        off0, nb = packed_range(self.shape, 0, max_layers)
        self.nbytes = off0 + nb
        dev = dw.packed.device
        self.slot = torch.empty(self.nbytes, dtype=torch.uint8, device=dev)
        self.host = torch.empty(self.nbytes, dtype=torch.uint8, pin_memory=True)
        self.host.copy_(dw.packed[:self.nbytes])
        self.slot[:off0].copy_(dw.packed[:off0])  # the shared LM head, once
        torch.cuda.current_stream().synchronize()
        self.event = Event()
        self.layers = 0  # layers whose load has been issued

    def load_async(self, n_layers: int, copy_stream=None) -> int:
        """Issue the H2D copy of layers [0, n_layers); returns the bytes sent."""
        if not 0 < n_layers <= self.max_layers:
            raise ValueError("n_layers outside the slot")
        off, nb = packed_range(self.shape, 0, n_layers)
        _check(lib().specdec_load_async(self.slot.data_ptr() + off, self.host.data_ptr() + off, nb,
                                        _stream(copy_stream), self.event.handle), "specdec_load_async")
        self.layers = n_layers
        return nb


# ---------------------------------------------------------------- entry points
def specdec_prefill(model: Model, kv: KVCache, tokens, stream=None):
    """tokens: device int32 [batch, n]."""
    import torch
    _dev(tokens, "tokens", torch.int32, kv.batch * tokens.shape[-1])
    if tokens.dim() != 2 or tokens.shape[0] != kv.batch:
        raise ValueError("tokens: expected [batch, n]")
    _check(lib().specdec_prefill(model.handle, ctypes.byref(kv.kv), tokens.shape[1], tokens.data_ptr(),
                                 _stream(stream)), "specdec_prefill")


def specdec_kv_append(kv: KVCache, layer: int, k, v, stream=None):
    """k, v: device bf16 [batch, n, n_kv_heads, head_dim]."""
    import torch
    shp = (kv.batch, k.shape[1] if k.dim() == 4 else 0, kv.kv.n_kv_heads, kv.kv.head_dim)
    for name, t in (("k", k), ("v", v)):
        _on_current(t, name, torch.bfloat16)
        _same_device(kv.data, "kv", t)
        if tuple(t.shape) != shp or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous [batch, n, {shp[2]}, {shp[3]}] tensor of one shape")
    _check(lib().specdec_kv_append(ctypes.byref(kv.kv), layer, shp[1], k.data_ptr(), v.data_ptr(), _stream(stream)),
           "specdec_kv_append")


def specdec_kv_advance(kv: KVCache, n: int, stream=None):
    import torch
    _on_current(kv.data, "kv", torch.uint8)
    _check(lib().specdec_kv_advance(ctypes.byref(kv.kv), n, _stream(stream)), "specdec_kv_advance")


class Rope:
    """The norm and position rotation of a model's heads (see specdec_rope).  ``rotary_dim``:
    dims that turn (all of them if not given); ``q_gain``, ``k_gain``: device
    tensors [head_dim], both float32 or both bfloat16, or None (no norm); ``freqs``: radians
    a position of every pair in place of base^(-2j / rotary_dim)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0,
                 interleaved: bool = False, q_gain=None, k_gain=None, eps: float = 1e-6, freqs=None):
        import torch
        gains = [g for g in (q_gain, k_gain) if g is not None]
        dtype = gains[0].dtype if gains else torch.float32
        for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
            if g is not None:
                _dev(g, name, dtype)
                _same_device(g, name, gains[0])
                if tuple(g.shape) != (head_dim,):
                    raise ValueError(f"{name}: expected [{head_dim}]")
        self.gains = (q_gain, k_gain)  # (kept alive with the rule)
        self.c = RopeDesc()
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        _check(lib().specdec_rope_init(ctypes.byref(self.c), head_dim, rotary_dim, base, int(interleaved),
                                       _ptr(q_gain), _ptr(k_gain), _float_type(dtype, "gains"), eps),
               "specdec_rope_init")
        if freqs is not None:
            freqs = [float(f) for f in freqs]
            if len(freqs) != rotary_dim // 2:
                raise ValueError(f"freqs: expected {rotary_dim // 2} entries")
            self.c.freq[:len(freqs)] = freqs
        self.ref = ctypes.byref(self.c)

    def _on(self, t):
        if self.gains[0] is not None:
            _same_device(t, "inputs", self.gains[0])
        elif self.gains[1] is not None:
            _same_device(t, "inputs", self.gains[1])


def _float_type(dtype, name: str) -> int:
    import torch
    if dtype == torch.bfloat16:
        return SPECDEC_BF16
    if dtype == torch.float32:
        return SPECDEC_F32
    raise ValueError(f"{name}: expected float32 or bfloat16, got {dtype}")


def _head_rows(t, name: str, head_dim: int, dtype=None):
    """The shape of t [batch, n, heads, head_dim], whose rows' heads lie side by side, and the stride between its rows."""
    _on_current(t, name, t.dtype if dtype is None else dtype)
    shape = t.shape
    if len(shape) != 4 or shape[3] != head_dim:
        raise ValueError(f"{name}: expected [batch, n, heads, {head_dim}]")
    if t.is_contiguous():
        return shape, shape[2] * head_dim
    stride = t.stride()
    if stride[3] != 1 or (shape[2] > 1 and stride[2] != head_dim):
        raise ValueError(f"{name}: a row's heads must lie side by side")
    width, one = shape[2] * head_dim, shape[0] == 1
    ld = stride[1] if shape[1] > 1 else width if one else stride[0]
    if ld >= width and (one or shape[1] == 1 or stride[0] == shape[1] * ld):
        return shape, ld
    return shape, _row_stride(t[:, :, 0], name, width)  # (raises)


def _positions(positions, rows, like):
    import torch
    if positions is None:
        return None
    if positions.shape != rows:
        raise ValueError(f"positions: expected {list(rows)}")
    _same_device(positions, "positions", like)
    return _dev(positions, "positions", torch.int32)


def specdec_rope_apply(rope: Rope, q, k, q_out, k_out, positions=None, offset: int = 0, stream=None):
    """q, q_out [batch, n, n_heads, head_dim], k, k_out [batch, n, n_kv_heads, head_dim], float32 or
    bfloat16 (inputs of one type, outputs of one), each with one stride between its rows; q and
    q_out, or k and k_out, may be None.  positions: int32 [batch, n] (0 .. n-1 if not given).
    An output may be its own input."""
    if (q is None and k is None) or (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("q, k: expected one of them at least, each with its output")
    some, to = (q, q_out) if q is not None else (k, k_out)
    hd, heads, lds = rope.c.head_dim, [], []
    rows = some.shape[:2]
    for name, t, out in (("q", q, q_out), ("k", k, k_out)):
        if t is None:
            heads.append(0)
            lds += [0, 0]
            continue
        shape, ld = _head_rows(t, name, hd, some.dtype)
        shape_out, ld_out = _head_rows(out, name + "_out", hd, to.dtype)
        if shape != shape_out or shape[:2] != rows:
            raise ValueError(f"{name}, {name}_out: expected one shape, of one batch of rows")
        heads.append(shape[2])
        lds += [ld, ld_out]
    rope._on(some)
    _check(lib().specdec_rope_apply(rope.ref, rows[0], rows[1], heads[0], heads[1], _float_type(some.dtype, "inputs"),
                                    _ptr(q), lds[0], _ptr(k), lds[2], _positions(positions, rows, some), offset,
                                    _float_type(to.dtype, "outputs"), _ptr(q_out), lds[1], _ptr(k_out), lds[3],
                                    _stream(stream)), "specdec_rope_apply")


def specdec_rope_append(kv: KVCache, layer: int, rope: Rope, q, k, v, q_out, positions=None, offset: int = 0,
                        stream=None):
    """q [batch, n, n_heads, head_dim], k, v [batch, n, n_kv_heads, head_dim], float32 or bfloat16, each
    with one stride between its rows; q_out: contiguous, of q's shape, float32 or
    bfloat16 (may be q).  positions: int32 [batch, n], the cache's own (offset + len[b] + i) if
    not given."""
    hd, G, B = kv.kv.head_dim, kv.kv.n_kv_heads, kv.kv.batch
    (shape, ld_q), (shape_k, ld_k), (shape_v, ld_v) = (_head_rows(t, name, hd, q.dtype)
                                                       for name, t in (("q", q), ("k", k), ("v", v)))
    n = shape[1]
    if shape[0] != B or shape_k != shape_v or shape_k != (B, n, G, hd):
        raise ValueError(f"q, k, v: expected rows of a batch of {B}, {G} kv heads")
    _on_current(q_out, "q_out", q_out.dtype)
    if q_out.shape != shape or not q_out.is_contiguous():
        raise ValueError("q_out: expected a contiguous tensor of q's shape")
    _same_device(kv.data, "kv", q)
    rope._on(q)
    _check(lib().specdec_rope_append(ctypes.byref(kv.kv), layer, rope.ref, n, shape[2],
                                     _float_type(q.dtype, "inputs"), q.data_ptr(), ld_q, k.data_ptr(), ld_k,
                                     v.data_ptr(), ld_v, _positions(positions, shape[:2], q), offset,
                                     _float_type(q_out.dtype, "q_out"), q_out.data_ptr(), _stream(stream)),
           "specdec_rope_append")


def attention_workspace(kv: KVCache, n_heads: int, n: int):
    """A device buffer large enough for specdec_attention's workspace."""
    import torch
    nbytes = lib().specdec_attention_workspace_bytes(ctypes.byref(kv.kv), n_heads, n)
    if nbytes == 0:
        raise ValueError("specdec_attention does not support this cache or these sizes")
    return torch.empty(nbytes, dtype=torch.uint8, device=kv.data.device)


def specdec_attention(kv: KVCache, layer: int, q, out, workspace=None, stream=None):
    """q, out: device float32 [batch, n, n_heads, head_dim] (out may be q).
    `workspace` (from attention_workspace) is allocated per call, on the call's stream, when
    not given.
    Calls on one cache must be ordered on one stream."""
    import torch
    if q.dim() != 4 or q.shape[0] != kv.batch or q.shape[3] != kv.kv.head_dim or out.shape != q.shape:
        raise ValueError("q, out: expected [batch, n, n_heads, head_dim]")
    for name, t in (("q", q), ("out", out)):
        _on_current(t, name, torch.float32)
        if not t.is_contiguous():
            raise ValueError(f"{name}: must be contiguous")
    _same_device(kv.data, "kv", q)
    n, n_heads = q.shape[1], q.shape[2]
    if workspace is None:
        with _memory_of(stream):
            workspace = attention_workspace(kv, n_heads, n)
    _dev(workspace, "workspace", torch.uint8, 1)
    _same_device(workspace, "workspace", q)
    _check(lib().specdec_attention(ctypes.byref(kv.kv), layer, n_heads, n, q.data_ptr(), out.data_ptr(),
                                   workspace.data_ptr(), workspace.numel(), _stream(stream)), "specdec_attention")


def shared_attention_workspace(prefix: KVCache, kv: KVCache, n_heads: int, n: int, dtype=None):
    """A device buffer large enough for specdec_attention_shared's workspace (dtype: of its
    queries, float32 if not given)."""
    import torch
    kind = SPECDEC_F32 if dtype is None else _float_type(dtype, "dtype")
    nbytes = lib().specdec_attention_shared_workspace_bytes(ctypes.byref(prefix.kv), ctypes.byref(kv.kv), n_heads, n,
                                                            kind)
    if nbytes == 0:
        raise ValueError("specdec_attention_shared does not support these caches or sizes")
    return torch.empty(nbytes, dtype=torch.uint8, device=kv.data.device)


def specdec_attention_shared(prefix: KVCache, kv: KVCache, layer: int, q, out, workspace=None, prefix_b: int = 0,
                             stream=None):
    """q, out: device float32 or bfloat16 [batch, n, n_heads, head_dim] (out may be q); `prefix`'s sequence
    `prefix_b` is what every sequence of `kv` begins with.
    `workspace` (from shared_attention_workspace) is allocated per call, on the call's stream,
    when not given.
    Calls on one `kv` must be ordered on one stream; `prefix` is only read."""
    import torch
    if q.dim() != 4 or q.shape[0] != kv.batch or q.shape[3] != kv.kv.head_dim or out.shape != q.shape:
        raise ValueError("q, out: expected [batch, n, n_heads, head_dim]")
    kind = _float_type(q.dtype, "q")
    for name, t in (("q", q), ("out", out)):
        _on_current(t, name, q.dtype)
        if not t.is_contiguous():
            raise ValueError(f"{name}: must be contiguous")
    _same_device(kv.data, "kv", q)
    _same_device(prefix.data, "prefix", q)
    n, n_heads = q.shape[1], q.shape[2]
    if workspace is None:
        with _memory_of(stream):
            workspace = shared_attention_workspace(prefix, kv, n_heads, n, q.dtype)
    _dev(workspace, "workspace", torch.uint8, 1)
    _same_device(workspace, "workspace", q)
    _check(lib().specdec_attention_shared(ctypes.byref(prefix.kv), prefix_b, ctypes.byref(kv.kv), layer, n_heads, n,
                                          kind, q.data_ptr(), out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                          _stream(stream)), "specdec_attention_shared")


def specdec_draft_step(draft: Model, kv: KVCache, gamma: int, slot: int, temperature: float, seed: int, step: int,
                       rand, q_out, d_out, ld_d: int, logits_out=None, stream=None, step_dev=None):
    """step_dev: a cache's KVCache.step_word() (device address of its commit
    counter) read in place of `step`, or None."""
    import torch
    B, V = kv.batch, draft.shape.vocab
    if rand is not None:
        _dev(rand, "rand", None, B)
        if rand.element_size() != 4:
            raise ValueError("rand: expected 32-bit words")
    _dev(q_out, "q_out", torch.float32, B * gamma * V, optional=temperature == 0)
    _dev(d_out, "d_out", torch.int32, (B - 1) * ld_d + gamma)
    _dev(logits_out, "logits_out", torch.float32, B * V, optional=True)
    _check(lib().specdec_draft_step(draft.handle, ctypes.byref(kv.kv), gamma, slot, temperature, seed, step,
                                    step_dev, _ptr(rand), _ptr(q_out), d_out.data_ptr(), ld_d, _ptr(logits_out),
                                    _stream(stream)), "specdec_draft_step")


def specdec_verify(target: Model, kv: KVCache, gamma: int, d, ld_d: int, logits_out, stream=None):
    import torch
    B, V = kv.batch, target.shape.vocab
    _dev(d, "d", torch.int32, (B - 1) * ld_d + gamma, optional=gamma == 0)
    _dev(logits_out, "logits_out", torch.float32, B * (gamma + 1) * V)
    _check(lib().specdec_verify(target.handle, ctypes.byref(kv.kv), gamma, _ptr(d), ld_d, logits_out.data_ptr(),
                                _stream(stream)), "specdec_verify")


def specdec_accept_workspace_bytes(batch: int, gamma: int, vocab: int) -> int:
    return int(lib().specdec_accept_workspace_bytes(batch, gamma, vocab))


def accept_workspace(batch: int, gamma: int, vocab: int, device="cuda"):
    """A device buffer large enough for specdec_accept's workspace."""
    import torch
    n = specdec_accept_workspace_bytes(batch, gamma, vocab)
    if n == 0:
        raise ValueError("specdec_accept does not support these sizes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def specdec_accept(batch: int, gamma: int, vocab: int, input_kind: int, temperature: float, p, q, d, ld_d: int,
                   rand, seed: int, step: int, n_accepted, next_token, status=None, workspace=None, stream=None,
                   step_dev=None):
    """Accept / resample.  `workspace` (uint8 device tensor) is allocated per
    call, on the call's stream, when not given; pass one from accept_workspace() in loops.  step_dev:
    as for specdec_draft_step."""
    import torch
    _dev(p, "p", torch.float32, batch * (gamma + 1) * vocab)
    _dev(q, "q", torch.float32, batch * gamma * vocab, optional=temperature == 0 or gamma == 0)
    _dev(d, "d", torch.int32, (batch - 1) * ld_d + gamma, optional=gamma == 0)
    if rand is not None:
        _dev(rand, "rand", rand.dtype, batch * (gamma + 1))
        if rand.dtype not in (torch.int32, torch.uint32):
            raise ValueError("rand: expected 32-bit words")
    _dev(n_accepted, "n_accepted", torch.int32, batch)
    _dev(next_token, "next_token", torch.int32, batch)
    _dev(status, "status", torch.int32, 1, optional=True)
    if workspace is None:
        with _memory_of(stream):
            workspace = accept_workspace(batch, gamma, vocab, p.device)
    _dev(workspace, "workspace", torch.uint8, 1)
    _check(lib().specdec_accept(batch, gamma, vocab, input_kind, temperature, p.data_ptr(), _ptr(q), _ptr(d), ld_d,
                                _ptr(rand), seed, step, step_dev, n_accepted.data_ptr(), next_token.data_ptr(),
                                _ptr(status), workspace.data_ptr(), workspace.numel(), _stream(stream)),
           "specdec_accept")


def specdec_accept_noalloc(batch: int, gamma: int, vocab: int, input_kind: int, temperature: float, p, q, d,
                           ld_d: int, rand, seed: int, step: int, n_accepted, next_token, status=None, stream=None,
                           step_dev=None):
    """specdec_accept with the library's static scratch (no workspace, no allocation)."""
    import torch
    _dev(p, "p", torch.float32, batch * (gamma + 1) * vocab)
    _dev(q, "q", torch.float32, batch * gamma * vocab, optional=temperature == 0 or gamma == 0)
    _dev(d, "d", torch.int32, (batch - 1) * ld_d + gamma, optional=gamma == 0)
    if rand is not None:
        _dev(rand, "rand", rand.dtype, batch * (gamma + 1))
        if rand.dtype not in (torch.int32, torch.uint32):
            raise ValueError("rand: expected 32-bit words")
    _dev(n_accepted, "n_accepted", torch.int32, batch)
    _dev(next_token, "next_token", torch.int32, batch)
    _dev(status, "status", torch.int32, 1, optional=True)
    _check(lib().specdec_accept_noalloc(batch, gamma, vocab, input_kind, temperature, p.data_ptr(), _ptr(q), _ptr(d),
                                        ld_d, _ptr(rand), seed, step, step_dev, n_accepted.data_ptr(),
                                        next_token.data_ptr(), _ptr(status), _stream(stream)),
           "specdec_accept_noalloc")


def specdec_kv_commit(kv: KVCache, gamma: int, role: int, n_accepted, d, ld_d: int, next_token, stream=None):
    import torch
    B = kv.batch
    _dev(n_accepted, "n_accepted", torch.int32, B)
    _dev(next_token, "next_token", torch.int32, B)
    _dev(d, "d", torch.int32, (B - 1) * ld_d + gamma, optional=role == ROLE_TARGET)
    _check(lib().specdec_kv_commit(ctypes.byref(kv.kv), gamma, role, n_accepted.data_ptr(), _ptr(d), ld_d,
                                   next_token.data_ptr(), _stream(stream)), "specdec_kv_commit")


def specdec_sample(probs, rand, seed: int, step: int, purpose: int, index: int, out, vocab=None, stream=None):
    import torch
    B, ld = probs.shape
    _dev(probs, "probs", torch.float32, B * ld)
    if rand is not None:
        _dev(rand, "rand", rand.dtype, B)
    _dev(out, "out", torch.int32, B)
    if vocab is not None and vocab > ld:
        raise ValueError("vocab > row length")
    _check(lib().specdec_sample(B, vocab or ld, probs.data_ptr(), ld, _ptr(rand), seed, step, purpose, index,
                                out.data_ptr(), _stream(stream)), "specdec_sample")


class SamplingRules:
    """Per-sequence sampling rules (see specdec_sampling): device tensors of one
    entry per sequence, float32 (top_k: int32), or None where a rule is off."""

    def __init__(self, temperature=None, top_k=None, top_p=None, min_p=None):
        import torch
        given = {"temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}
        self.tensors = {k: t for k, t in given.items() if t is not None}
        sizes = set()
        for k, t in self.tensors.items():
            _dev(t, k, torch.int32 if k == "top_k" else torch.float32, 1)
            sizes.add(t.numel())
        if len(sizes) > 1:
            raise ValueError("rules: one entry per sequence in each tensor")
        self.batch = sizes.pop() if sizes else None
        self.c = Sampling(*[_ptr(given[k]) for k in ("temperature", "top_k", "top_p", "min_p")])


def sample_workspace(batch: int, rows: int, vocab: int, device="cuda"):
    """A device buffer large enough for specdec_sample_logits' workspace."""
    import torch
    n = lib().specdec_sample_logits_workspace_bytes(batch, rows, vocab)
    if n == 0:
        raise ValueError("specdec_sample_logits does not support these sizes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def specdec_sample_logits(logits, rules: Optional[SamplingRules] = None, rand=None, seed: int = 0, step: int = 0,
                          purpose: int = PURPOSE_RESAMPLE, index: int = 0, probs=None, out=None, status=None,
                          workspace=None, stream=None, step_dev=None):
    """logits [batch, rows, vocab] or [batch, vocab] float32; probs: the same
    shape; out: int32 [batch, rows].  probs and out may be strided over their
    leading dimensions (a slot of a larger buffer) if one stride covers them.
    `workspace` is allocated per call, on the call's stream, when not given."""
    import torch
    _on_current(logits, "logits", torch.float32)
    if logits.dim() not in (2, 3):
        raise ValueError("logits: expected [batch, rows, vocab] or [batch, vocab]")
    batch, vocab = logits.shape[0], logits.shape[-1]
    rows = logits.shape[1] if logits.dim() == 3 else 1
    ld = _row_stride(logits, "logits", vocab)
    if rules is not None:
        if rules.batch is not None and rules.batch != batch:
            raise ValueError(f"rules: {rules.batch} entries for a batch of {batch}")
        for k, t in rules.tensors.items():
            _same_device(t, k, logits)
    if rand is not None:
        _dev(rand, "rand", None, batch * rows)
        if rand.dtype not in (torch.int32, torch.uint32):
            raise ValueError("rand: expected 32-bit words")
        _same_device(rand, "rand", logits)
    ld_probs = ld_out = 0
    if probs is not None:
        if probs.shape != logits.shape:
            raise ValueError("probs: expected the shape of logits")
        _on_current(probs, "probs", torch.float32)
        ld_probs = _row_stride(probs, "probs", vocab)
    if out is not None:
        if out.numel() != batch * rows:
            raise ValueError("out: expected one entry per row")
        _on_current(out, "out", torch.int32)
        ld_out = _row_stride(out.reshape(batch, rows, 1) if out.is_contiguous() else out.unsqueeze(-1), "out", 1)
    if status is not None:
        _dev(status, "status", torch.int32, 1)
        _same_device(status, "status", logits)
    if workspace is None:
        with _memory_of(stream):
            workspace = sample_workspace(batch, rows, vocab, logits.device)
    _dev(workspace, "workspace", torch.uint8, 1)
    _same_device(workspace, "workspace", logits)
    _check(lib().specdec_sample_logits(batch, rows, vocab, logits.data_ptr(), ld,
                                       None if rules is None else ctypes.byref(rules.c), _ptr(rand), seed, step,
                                       step_dev, purpose, index, _ptr(probs), ld_probs, _ptr(out), ld_out,
                                       _ptr(status), workspace.data_ptr(), workspace.numel(), _stream(stream)),
           "specdec_sample_logits")


def _on_current(t, name: str, dtype):
    """Check a tensor argument's type, and that it is on the current device (where the call launches)."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


def _same_device(t, name: str, other):
    if t.device != other.device:
        raise ValueError(f"{name}: on {t.device}, expected {other.device}")


def _row_stride(t, name: str, width: int) -> int:
    """The one stride between the rows of t [batch, rows, width] (or [batch, width])."""
    if width > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    lead = [(n, s) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n > 1]
    if not lead:
        return width
    ld = lead[-1][1]
    for (_, s), (n1, s1) in zip(lead[:-1], lead[1:]):
        if s != n1 * s1:
            raise ValueError(f"{name}: rows need one stride")
    if ld < width:
        raise ValueError(f"{name}: rows overlap")
    return ld


def specdec_draw_u32(batch: int, seed: int, step: int, purpose: int, index: int, out, stream=None):
    _dev(out, "out", out.dtype if out is not None else None, batch)
    if out.element_size() != 4:
        raise ValueError("out: expected 32-bit words")
    _check(lib().specdec_draw_u32(batch, seed, step, purpose, index, out.data_ptr(), _stream(stream)),
           "specdec_draw_u32")


def specdec_device_status(kv: KVCache, stream=None) -> int:
    out = ctypes.c_int32(0)
    lib().specdec_device_status(ctypes.byref(kv.kv), _stream(stream), ctypes.byref(out))
    return out.value


def specdec_stream_read(buf, sink, nbytes=None, stream=None):
    """Streaming-read ceiling probe over a device tensor (see the header)."""
    _dev(buf, "buf", None, 1)
    _dev(sink, "sink", None, 1)
    size = buf.numel() * buf.element_size()
    n = size if nbytes is None else int(nbytes)
    if not 0 <= n <= size:
        raise ValueError("nbytes: outside the buffer")
    _check(lib().specdec_stream_read(buf.data_ptr(), n, sink.data_ptr(), _stream(stream)), "specdec_stream_read")


def specdec_status_string(status: int) -> str:
    return lib().specdec_status_string(status).decode()


def specdec_timing_enable(enable: bool):
    _check(lib().specdec_timing_enable(1 if enable else 0), "specdec_timing_enable")


def specdec_time_kernel(model: "Model", kind: str, reps: int = 20, stream=None) -> float:
    """Average duration (us) of `kind` re-launched back to back, layer after layer (see the header)."""
    out = ctypes.c_double(0.0)
    _check(lib().specdec_time_kernel(model.handle, KERNEL_KINDS.index(kind), reps, _stream(stream),
                                     ctypes.byref(out)), "specdec_time_kernel")
    return out.value


def specdec_timing_read():
    """{kind: (total_ms, launches)} since the last read (synchronizes on the events)."""
    ms = np.zeros(len(KERNEL_KINDS), np.float64)
    n = np.zeros(len(KERNEL_KINDS), np.int64)
    _check(lib().specdec_timing_read(ms.ctypes.data, n.ctypes.data), "specdec_timing_read")
    return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(KERNEL_KINDS)}


# ---------------------------------------------------------------- one iteration
class SpecDecoder:
    """Buffers and call sequence of one draft-and-verify iteration for a batch.

    The call order is the inner loop of the paper's runtime (Sec. 3.4, Alg. 3):
    gamma draft steps, one verify pass, accept / resample, commit of both
    caches.  Host code only sequences the calls; tokens and counts stay on
    the device.  With device_step the Philox step of every draw is the target
    cache's commit counter, read on the device (the `step` arguments below are
    then ignored), so a captured iteration draws fresh words on each replay.
    With ``rules`` (per-sequence SamplingRules, one entry per sequence; their
    temperatures take the place of ``temperature``) the draft proposes from the
    distribution the rules leave of its logits, and the accept tests it against
    the one they leave of the target's: the emitted tokens are distributed as
    sampling from the target under the rules.
    """

    def __init__(self, target: Model, draft: Model, kv_t: KVCache, kv_d: KVCache, gamma: int,
                 temperature: float, seed: int, device_step: bool = False, rules: Optional[SamplingRules] = None):
        import torch
        self.target, self.draft, self.kv_t, self.kv_d = target, draft, kv_t, kv_d
        self.gamma, self.temperature, self.seed = gamma, temperature, seed
        self.step_dev = kv_t.step_word() if device_step else None
        B, V = kv_t.batch, target.shape.vocab
        dev = kv_t.data.device
        self.B, self.V = B, V
        self.d = torch.zeros((B, gamma), dtype=torch.int32, device=dev)
        self.rules = rules
        if rules is not None and rules.batch not in (None, B):
            raise ValueError(f"rules: {rules.batch} entries for a batch of {B}")
        sampled = temperature > 0 or rules is not None
        self.q = torch.zeros((B, gamma, V), dtype=torch.float32, device=dev) if sampled else None
        self.logits = torch.empty((B, gamma + 1, V), dtype=torch.float32, device=dev)
        self.n_acc = torch.zeros(B, dtype=torch.int32, device=dev)
        self.next = torch.zeros(B, dtype=torch.int32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.accept_ws = accept_workspace(B, gamma, V, dev)
        if rules is not None:
            self.p = torch.empty((B, gamma + 1, V), dtype=torch.float32, device=dev)
            self.draft_logits = torch.empty((B, V), dtype=torch.float32, device=dev)
            self.rules_ws = sample_workspace(B, gamma + 1, V, dev)

    def draft_phase(self, step: int, stream=None):
        for s in range(self.gamma):
            if self.rules is not None:
                specdec_draft_step(self.draft, self.kv_d, self.gamma, s, 0.0, self.seed, step, None, None, self.d,
                                   self.gamma, self.draft_logits, stream, step_dev=self.step_dev)
                specdec_sample_logits(self.draft_logits, self.rules, seed=self.seed, step=step, purpose=PURPOSE_DRAFT,
                                      index=s, probs=self.q[:, s], out=self.d[:, s], status=self.status,
                                      workspace=self.rules_ws, stream=stream, step_dev=self.step_dev)
                continue
            specdec_draft_step(self.draft, self.kv_d, self.gamma, s, self.temperature, self.seed, step, None, self.q,
                               self.d, self.gamma, None, stream, step_dev=self.step_dev)

    def verify_phase(self, step: int, stream=None):
        specdec_verify(self.target, self.kv_t, self.gamma, self.d, self.gamma, self.logits, stream)
        kind, temperature, scores = INPUT_LOGITS, self.temperature, self.logits
        if self.rules is not None:
            specdec_sample_logits(self.logits, self.rules, probs=self.p, status=self.status, workspace=self.rules_ws,
                                  stream=stream)
            kind, temperature, scores = INPUT_PROBS, 1.0, self.p
        specdec_accept(self.B, self.gamma, self.V, kind, temperature, scores, self.q, self.d,
                       self.gamma, None, self.seed, step, self.n_acc, self.next, self.status, self.accept_ws, stream,
                       step_dev=self.step_dev)

    def commit_phase(self, stream=None):
        specdec_kv_commit(self.kv_t, self.gamma, ROLE_TARGET, self.n_acc, self.d, self.gamma, self.next, stream)
        specdec_kv_commit(self.kv_d, self.gamma, ROLE_DRAFT, self.n_acc, self.d, self.gamma, self.next, stream)

    def step(self, step: int, stream=None):
        self.draft_phase(step, stream)
        self.verify_phase(step, stream)
        self.commit_phase(stream)
