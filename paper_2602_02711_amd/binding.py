"""Python binding of ``include/dmr_qlinear.h``: argument marshalling only.

Every function has the name and meaning of the C entry point it calls; tensors are torch
tensors used as device memory (PyTorch supplies allocation and streams, nothing else) and all
arithmetic happens in the HIP kernels of ``libdmr_qlinear.so``.  There is no fallback: if the
library is missing or a call is refused, an exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdmr_qlinear.so")

DMR_OK = 0
DMR_ERR_NULL, DMR_ERR_SHAPE, DMR_ERR_ALIGN, DMR_ERR_WORKSPACE, DMR_ERR_UNSUPPORTED, DMR_ERR_HIP = range(1, 7)
DMR_OUT_BF16, DMR_OUT_FP32 = 0, 1

EXPORTS = (
    "dmr_qlinear_storage_bytes", "dmr_qlinear_workspace_bytes", "dmr_qlinear_bf16_workspace_bytes",
    "dmr_qlinear_create",
    "dmr_qlinear_dequantize", "dmr_qlinear_forward", "dmr_qlinear_bf16_forward",
    "dmr_qlinear_quantize", "dmr_qlinear_destroy", "dmr_qlinear_shape", "dmr_status_string",
    "dmr_probe_hbm_read", "dmr_qlinear_w3_storage_bytes", "dmr_qlinear_w3_workspace_bytes",
    "dmr_qlinear_w3_create", "dmr_qlinear_quantize_w3", "dmr_qlinear_bits", "dmr_qlinear_create_per_channel",
    "dmr_glue_rmsnorm", "dmr_glue_swiglu", "dmr_qlinear_fused_workspace_bytes",
    "dmr_qlinear_bf16_fused_workspace_bytes", "dmr_qlinear_forward_fused", "dmr_qlinear_bf16_forward_fused",
    "dmr_qlinear_kernel_path", "dmr_qlinear_forward_static", "dmr_probe_empty_launch",
    "dmr_qlinear_per_channel_storage_bytes",
    "dmr_kv_page_bytes", "dmr_kv_assign", "dmr_kv_append", "dmr_attn_paged_workspace_bytes", "dmr_attn_paged",
)

DMR_PRO_NONE, DMR_PRO_RMSNORM, DMR_PRO_SWIGLU = 0, 1, 2
DMR_FMT_W4_G128, DMR_FMT_W4_PER_CHANNEL, DMR_FMT_W3_G128, DMR_FMT_BF16 = 0, 1, 2, 3
DMR_KV_BF16, DMR_KV_E4M3 = 0, 1
DMR_ROPE_HALVES, DMR_ROPE_ADJACENT = 0, 1


class _KvCacheStruct(ctypes.Structure):
    """dmr_kv_cache_t"""
    _fields_ = [("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_tokens", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("type", ctypes.c_int), ("k_scale", ctypes.c_float),
                ("v_scale", ctypes.c_float)]


class DmrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        text = lib().dmr_status_string(status).decode()
        super().__init__(f"{where}: {text} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library, with prototypes set.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
        L.dmr_qlinear_storage_bytes.restype = sz
        L.dmr_qlinear_storage_bytes.argtypes = [i64, i64, i32]
        L.dmr_qlinear_workspace_bytes.restype = sz
        L.dmr_qlinear_workspace_bytes.argtypes = [i64, i64, i64]
        L.dmr_qlinear_bf16_workspace_bytes.restype = sz
        L.dmr_qlinear_bf16_workspace_bytes.argtypes = [i64, i64, i64]
        L.dmr_qlinear_create.restype = ctypes.c_int
        L.dmr_qlinear_create.argtypes = [ctypes.POINTER(vp), i64, i64, i32, vp, vp, vp, vp, sz, vp]
        L.dmr_qlinear_dequantize.restype = ctypes.c_int
        L.dmr_qlinear_dequantize.argtypes = [vp, vp, vp]
        L.dmr_qlinear_forward.restype = ctypes.c_int
        L.dmr_qlinear_forward.argtypes = [vp, vp, i64, vp, ctypes.c_int, vp, sz, vp]
        L.dmr_qlinear_forward_static.restype = ctypes.c_int
        L.dmr_qlinear_forward_static.argtypes = [vp, vp, i64, vp, ctypes.c_int, vp]
        L.dmr_qlinear_bf16_forward.restype = ctypes.c_int
        L.dmr_qlinear_bf16_forward.argtypes = [vp, vp, i64, i64, i64, vp, ctypes.c_int, vp, sz, vp]
        L.dmr_qlinear_quantize.restype = ctypes.c_int
        L.dmr_qlinear_quantize.argtypes = [i64, i64, i32, vp, vp, vp, vp, vp]
        L.dmr_qlinear_destroy.restype = None
        L.dmr_qlinear_destroy.argtypes = [vp]
        L.dmr_qlinear_shape.restype = ctypes.c_int
        L.dmr_qlinear_shape.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i32)]
        L.dmr_qlinear_w3_storage_bytes.restype = sz
        L.dmr_qlinear_w3_storage_bytes.argtypes = [i64, i64, i32]
        L.dmr_qlinear_w3_workspace_bytes.restype = sz
        L.dmr_qlinear_w3_workspace_bytes.argtypes = [i64, i64, i64]
        L.dmr_qlinear_w3_create.restype = ctypes.c_int
        L.dmr_qlinear_w3_create.argtypes = [ctypes.POINTER(vp), i64, i64, i32, vp, vp, vp, vp, sz, vp]
        L.dmr_qlinear_quantize_w3.restype = ctypes.c_int
        L.dmr_qlinear_quantize_w3.argtypes = [i64, i64, i32, vp, vp, vp, vp, vp]
        L.dmr_qlinear_per_channel_storage_bytes.restype = sz
        L.dmr_qlinear_per_channel_storage_bytes.argtypes = [i64, i64]
        L.dmr_qlinear_create_per_channel.restype = ctypes.c_int
        L.dmr_qlinear_create_per_channel.argtypes = [ctypes.POINTER(vp), i64, i64, vp, vp, vp, sz, vp]
        L.dmr_qlinear_bits.restype = i32
        L.dmr_qlinear_bits.argtypes = [vp]
        L.dmr_probe_empty_launch.restype = ctypes.c_int
        L.dmr_probe_empty_launch.argtypes = [i32, i32, sz, vp]
        L.dmr_probe_hbm_read.restype = ctypes.c_int
        L.dmr_probe_hbm_read.argtypes = [vp, sz, vp, i32, vp]
        f32 = ctypes.c_float
        L.dmr_glue_rmsnorm.restype = ctypes.c_int
        L.dmr_glue_rmsnorm.argtypes = [vp, vp, f32, i64, i64, vp, vp]
        L.dmr_glue_swiglu.restype = ctypes.c_int
        L.dmr_glue_swiglu.argtypes = [vp, i64, i64, vp, vp]
        L.dmr_qlinear_fused_workspace_bytes.restype = sz
        L.dmr_qlinear_fused_workspace_bytes.argtypes = [vp, i64, ctypes.c_int, i32]
        L.dmr_qlinear_bf16_fused_workspace_bytes.restype = sz
        L.dmr_qlinear_bf16_fused_workspace_bytes.argtypes = [i64, i64, i64, ctypes.c_int, i32]
        L.dmr_qlinear_forward_fused.restype = ctypes.c_int
        L.dmr_qlinear_forward_fused.argtypes = [vp, ctypes.c_int, vp, vp, f32, vp, i64, vp, ctypes.c_int, vp, sz, vp]
        L.dmr_qlinear_bf16_forward_fused.restype = ctypes.c_int
        L.dmr_qlinear_bf16_forward_fused.argtypes = [vp, ctypes.c_int, vp, vp, f32, vp, i64, i64, i64, vp,
                                                     ctypes.c_int, vp, sz, vp]
        cache = ctypes.POINTER(_KvCacheStruct)
        L.dmr_kv_page_bytes.restype = sz
        L.dmr_kv_page_bytes.argtypes = [i32, i32, i32, ctypes.c_int]
        L.dmr_kv_assign.restype = ctypes.c_int
        L.dmr_kv_assign.argtypes = [i64, i64, i64, i32, i64] + [vp] * 11
        L.dmr_kv_append.restype = ctypes.c_int
        L.dmr_kv_append.argtypes = [cache, vp, i64, i32, vp, vp, f32, vp, ctypes.c_int, vp, vp, vp, vp]
        L.dmr_attn_paged_workspace_bytes.restype = sz
        L.dmr_attn_paged_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i64]
        L.dmr_attn_paged.restype = ctypes.c_int
        L.dmr_attn_paged.argtypes = [cache, vp, i64, i32, i64, vp, vp, vp, i64, i64, f32, vp, vp, sz, vp]
        L.dmr_status_string.restype = ctypes.c_char_p
        L.dmr_status_string.argtypes = [ctypes.c_int]
        L.dmr_qlinear_kernel_path.restype = ctypes.c_char_p
        L.dmr_qlinear_kernel_path.argtypes = [ctypes.c_int, i64, i64, i64]
        _lib = L
    return _lib


def _check(status: int, where: str) -> None:
    if status != DMR_OK:
        raise DmrError(status, where)


def _dev(t: torch.Tensor, name: str, dtypes) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a tensor in device memory")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)
_U32 = (torch.int32, torch.uint32)


def _stream(stream) -> int:
    if stream is None:
        # the current device's current stream, without the Stream object that torch.cuda.current_stream() makes (2.8 us / 0.2
        # of a call of 10)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _output(out, M: int, N: int, dtype, like: torch.Tensor):
    """(out or a new tensor, its address)"""
    if out is None:
        _out_code(dtype)
        out = torch.empty((M, N), dtype=dtype, device=like.device)
        return out, out.data_ptr()
    po = _dev(out, "out", (torch.bfloat16, torch.float32))
    if tuple(out.shape) != (M, N):
        raise ValueError("out must be [M][N]")
    return out, po


def _out_code(dtype) -> int:
    if dtype == torch.bfloat16:
        return DMR_OUT_BF16
    if dtype == torch.float32:
        return DMR_OUT_FP32
    raise TypeError("output dtype must be torch.bfloat16 or torch.float32")


class Layer:
    """Host handle of one quantised Linear layer plus the storage tensor it points into."""

    def __init__(self, handle: int, storage: torch.Tensor, K: int, N: int, g: int, bits: int = 4):
        self.handle, self.storage, self.K, self.N, self.g, self.bits = handle, storage, K, N, g, bits

    def __del__(self):
        dmr_qlinear_destroy(self)


def dmr_qlinear_storage_bytes(K: int, N: int, g: int = 128) -> int:
    return int(lib().dmr_qlinear_storage_bytes(K, N, g))


def dmr_qlinear_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(lib().dmr_qlinear_workspace_bytes(M, K, N))


def dmr_qlinear_bf16_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(lib().dmr_qlinear_bf16_workspace_bytes(M, K, N))


def dmr_qlinear_create(qweight: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, g: int = 128,
                       storage: torch.Tensor | None = None, stream=None) -> Layer:
    pq = _dev(qweight, "qweight", _U32)
    ps = _dev(scales, "scales", _BF16)
    pz = _dev(zeros, "zeros", _BF16)
    N, K8 = qweight.shape
    K = K8 * 8
    if g <= 0 or K % g or tuple(scales.shape) != (N, K // g) or tuple(zeros.shape) != (N, K // g):
        raise ValueError("scales and zeros must be [N][K/g]")
    need = dmr_qlinear_storage_bytes(K, N, g)
    if storage is None:
        storage = torch.empty(max(need, 16), dtype=torch.uint8, device=qweight.device)
    pst = _dev(storage, "storage", (torch.uint8,))
    handle = ctypes.c_void_p()
    _check(lib().dmr_qlinear_create(ctypes.byref(handle), K, N, g, pq, ps, pz, pst, storage.numel(),
                                    _stream(stream)), "dmr_qlinear_create")
    return Layer(handle.value, storage, K, N, g)


def dmr_qlinear_dequantize(layer: Layer, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((layer.N, layer.K), dtype=torch.bfloat16, device=layer.storage.device)
    po = _dev(out, "out", _BF16)
    if tuple(out.shape) != (layer.N, layer.K):
        raise ValueError("out must be [N][K]")
    _check(lib().dmr_qlinear_dequantize(layer.handle, po, _stream(stream)), "dmr_qlinear_dequantize")
    return out


def _workspace(workspace):
    if workspace is None:
        return None, 0
    return _dev(workspace, "workspace", (torch.uint8,)), workspace.numel()


def dmr_qlinear_forward(layer: Layer, x: torch.Tensor, out: torch.Tensor | None = None,
                        out_dtype=torch.bfloat16, workspace: torch.Tensor | None = None,
                        stream=None) -> torch.Tensor:
    px = _dev(x, "x", _BF16)
    if x.dim() != 2 or x.shape[1] != layer.K:
        raise ValueError("x must be [M][K]")
    M = x.shape[0]
    out, po = _output(out, M, layer.N, out_dtype, x)
    need = (dmr_qlinear_w3_workspace_bytes(M, layer.K, layer.N) if layer.bits == 3
            else dmr_qlinear_workspace_bytes(M, layer.K, layer.N))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)    # device memory only
    pw, wbytes = _workspace(workspace)
    _check(lib().dmr_qlinear_forward(layer.handle, px, M, po, _out_code(out.dtype), pw, wbytes,
                                     _stream(stream)), "dmr_qlinear_forward")
    return out


DMR_STATIC_SCRATCH_BYTES = 8 << 20


def dmr_qlinear_forward_static(layer: Layer, x: torch.Tensor, out: torch.Tensor | None = None,
                               out_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """dmr_qlinear_forward on the library's own fixed scratch: no workspace is passed or allocated."""
    px = _dev(x, "x", _BF16)
    if x.dim() != 2 or x.shape[1] != layer.K:
        raise ValueError("x must be [M][K]")
    M = x.shape[0]
    out, po = _output(out, M, layer.N, out_dtype, x)
    _check(lib().dmr_qlinear_forward_static(layer.handle, px, M, po, _out_code(out.dtype), _stream(stream)),
           "dmr_qlinear_forward_static")
    return out


def dmr_qlinear_bf16_forward(w: torch.Tensor, x: torch.Tensor, out: torch.Tensor | None = None,
                             out_dtype=torch.bfloat16, workspace: torch.Tensor | None = None,
                             stream=None) -> torch.Tensor:
    pw_ = _dev(w, "w", _BF16)
    px = _dev(x, "x", _BF16)
    N, K = w.shape
    if x.dim() != 2 or x.shape[1] != K:
        raise ValueError("x must be [M][K]")
    M = x.shape[0]
    out, po = _output(out, M, N, out_dtype, x)
    if workspace is None:
        need = dmr_qlinear_bf16_workspace_bytes(M, K, N)
        if need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)    # device memory only
    pws, wbytes = _workspace(workspace)
    _check(lib().dmr_qlinear_bf16_forward(pw_, px, M, K, N, po, _out_code(out.dtype), pws, wbytes,
                                          _stream(stream)), "dmr_qlinear_bf16_forward")
    return out


def dmr_qlinear_quantize(w: torch.Tensor, g: int = 128, stream=None):
    """fp32 [N][K] in device memory -> (qweight int32 [N][K/8], scales bf16, zeros bf16 [N][K/g])."""
    pw_ = _dev(w, "w", (torch.float32,))
    N, K = w.shape
    if g <= 0 or K % g or K % 8:
        raise ValueError("K must be a multiple of g and of 8")
    qweight = torch.empty((N, K // 8), dtype=torch.int32, device=w.device)
    scales = torch.empty((N, K // g), dtype=torch.bfloat16, device=w.device)
    zeros = torch.empty((N, K // g), dtype=torch.bfloat16, device=w.device)
    _check(lib().dmr_qlinear_quantize(K, N, g, pw_, qweight.data_ptr(), scales.data_ptr(),
                                      zeros.data_ptr(), _stream(stream)), "dmr_qlinear_quantize")
    return qweight, scales, zeros


def dmr_qlinear_per_channel_storage_bytes(K: int, N: int) -> int:
    return int(lib().dmr_qlinear_per_channel_storage_bytes(K, N))


def dmr_qlinear_create_per_channel(qweight: torch.Tensor, scales: torch.Tensor,
                                   storage: torch.Tensor | None = None, stream=None) -> Layer:
    """Symmetric per-channel INT4: qweight [N][K/8], one bf16 scale per row, zero point 8."""
    pq = _dev(qweight, "qweight", _U32)
    ps = _dev(scales, "scales", _BF16)
    N, K8 = qweight.shape
    K = K8 * 8
    if scales.numel() != N:
        raise ValueError("scales must hold one value per row")
    need = dmr_qlinear_per_channel_storage_bytes(K, N)
    if storage is None:
        storage = torch.empty(max(need, 16), dtype=torch.uint8, device=qweight.device)
    pst = _dev(storage, "storage", (torch.uint8,))
    handle = ctypes.c_void_p()
    _check(lib().dmr_qlinear_create_per_channel(ctypes.byref(handle), K, N, pq, ps, pst, storage.numel(),
                                                _stream(stream)), "dmr_qlinear_create_per_channel")
    return Layer(handle.value, storage, K, N, K)


def dmr_qlinear_w3_storage_bytes(K: int, N: int, g: int = 128) -> int:
    return int(lib().dmr_qlinear_w3_storage_bytes(K, N, g))


def dmr_qlinear_w3_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(lib().dmr_qlinear_w3_workspace_bytes(M, K, N))


def dmr_qlinear_w3_create(qweight3: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, g: int = 128,
                          storage: torch.Tensor | None = None, stream=None) -> Layer:
    pq = _dev(qweight3, "qweight3", _U32)
    ps = _dev(scales, "scales", _BF16)
    pz = _dev(zeros, "zeros", _BF16)
    N, W = qweight3.shape
    if W % 3:
        raise ValueError("qweight3 must be [N][3K/32]")
    K = W // 3 * 32
    if g <= 0 or K % g or tuple(scales.shape) != (N, K // g) or tuple(zeros.shape) != (N, K // g):
        raise ValueError("scales and zeros must be [N][K/g]")
    need = dmr_qlinear_w3_storage_bytes(K, N, g)
    if storage is None:
        storage = torch.empty(max(need, 16), dtype=torch.uint8, device=qweight3.device)
    pst = _dev(storage, "storage", (torch.uint8,))
    handle = ctypes.c_void_p()
    _check(lib().dmr_qlinear_w3_create(ctypes.byref(handle), K, N, g, pq, ps, pz, pst, storage.numel(),
                                       _stream(stream)), "dmr_qlinear_w3_create")
    return Layer(handle.value, storage, K, N, g, bits=3)


def dmr_qlinear_quantize_w3(w: torch.Tensor, g: int = 128, stream=None):
    """fp32 [N][K] in device memory -> (qweight3 int32 [N][3K/32], scales bf16, zeros bf16 [N][K/g])."""
    pw_ = _dev(w, "w", (torch.float32,))
    N, K = w.shape
    if g <= 0 or K % g or K % 32:
        raise ValueError("K must be a multiple of g and of 32")
    qweight = torch.empty((N, K // 32 * 3), dtype=torch.int32, device=w.device)
    scales = torch.empty((N, K // g), dtype=torch.bfloat16, device=w.device)
    zeros = torch.empty((N, K // g), dtype=torch.bfloat16, device=w.device)
    _check(lib().dmr_qlinear_quantize_w3(K, N, g, pw_, qweight.data_ptr(), scales.data_ptr(),
                                         zeros.data_ptr(), _stream(stream)), "dmr_qlinear_quantize_w3")
    return qweight, scales, zeros


def dmr_probe_hbm_read(buf: torch.Tensor, sink: torch.Tensor, blocks: int, stream=None) -> None:
    pb = _dev(buf, "buf", (torch.uint8,))
    ps = _dev(sink, "sink", (torch.int32, torch.uint32))
    if sink.numel() < blocks * 256:
        raise ValueError("sink needs blocks * 256 words")
    _check(lib().dmr_probe_hbm_read(pb, buf.numel(), ps, blocks, _stream(stream)), "dmr_probe_hbm_read")


def dmr_probe_empty_launch(blocks: int, threads: int, lds_bytes: int = 0, stream=None) -> None:
    _check(lib().dmr_probe_empty_launch(blocks, threads, lds_bytes, _stream(stream)), "dmr_probe_empty_launch")


def dmr_qlinear_kernel_path(fmt: int, M: int, K: int, N: int) -> str:
    return lib().dmr_qlinear_kernel_path(fmt, M, K, N).decode()


def dmr_qlinear_destroy(layer: Layer) -> None:
    handle, layer.handle = getattr(layer, "handle", None), None
    if handle and _lib is not None:
        _lib.dmr_qlinear_destroy(handle)


# ---- decoder glue and fused forwards -------------------------------------------------------------

def dmr_glue_rmsnorm(x: torch.Tensor, gamma: torch.Tensor, eps: float, out: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    px, pg = _dev(x, "x", _BF16), _dev(gamma, "gamma", _BF16)
    M, K = x.shape
    if tuple(gamma.shape) != (K,):
        raise ValueError("gamma must be [K]")
    if out is None:
        out = torch.empty((M, K), dtype=torch.bfloat16, device=x.device)
    po = _dev(out, "out", _BF16)
    _check(lib().dmr_glue_rmsnorm(px, pg, float(eps), M, K, po, _stream(stream)), "dmr_glue_rmsnorm")
    return out


def dmr_glue_swiglu(gate_up: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    pi = _dev(gate_up, "gate_up", _BF16)
    M, two_i = gate_up.shape
    if two_i % 2:
        raise ValueError("gate_up must be [M][2 I]")
    if out is None:
        out = torch.empty((M, two_i // 2), dtype=torch.bfloat16, device=gate_up.device)
    po = _dev(out, "out", _BF16)
    _check(lib().dmr_glue_swiglu(pi, M, two_i // 2, po, _stream(stream)), "dmr_glue_swiglu")
    return out


def _fused_args(pro, inp, gamma, residual, K, N):
    pi = _dev(inp, "inp", _BF16)
    want = 2 * K if pro == DMR_PRO_SWIGLU else K
    if inp.dim() != 2 or inp.shape[1] != want:
        raise ValueError(f"inp must be [M][{want}]")
    M = inp.shape[0]
    pg = None
    if pro == DMR_PRO_RMSNORM:
        pg = _dev(gamma, "gamma", _BF16)
        if tuple(gamma.shape) != (K,):
            raise ValueError("gamma must be [K]")
    pr = None
    if residual is not None:
        pr = _dev(residual, "residual", _BF16)
        if tuple(residual.shape) != (M, N):
            raise ValueError("residual must be [M][N]")
    return pi, pg, pr, M


def dmr_qlinear_forward_fused(layer: Layer, pro: int, inp: torch.Tensor, gamma: torch.Tensor | None = None,
                              eps: float = 0.0, residual: torch.Tensor | None = None,
                              out: torch.Tensor | None = None, out_dtype=torch.bfloat16,
                              workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    pi, pg, pr, M = _fused_args(pro, inp, gamma, residual, layer.K, layer.N)
    out, po = _output(out, M, layer.N, out_dtype, inp)
    if workspace is None:
        need = int(lib().dmr_qlinear_fused_workspace_bytes(layer.handle, M, pro, 1 if residual is not None else 0))
        if need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=inp.device)    # device memory only
    pw, wbytes = _workspace(workspace)
    _check(lib().dmr_qlinear_forward_fused(layer.handle, pro, pi, pg, float(eps), pr, M, po, _out_code(out.dtype),
                                           pw, wbytes, _stream(stream)), "dmr_qlinear_forward_fused")
    return out


def dmr_qlinear_bf16_forward_fused(w: torch.Tensor, pro: int, inp: torch.Tensor, gamma: torch.Tensor | None = None,
                                   eps: float = 0.0, residual: torch.Tensor | None = None,
                                   out: torch.Tensor | None = None, out_dtype=torch.bfloat16,
                                   workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    pw_ = _dev(w, "w", _BF16)
    N, K = w.shape
    pi, pg, pr, M = _fused_args(pro, inp, gamma, residual, K, N)
    out, po = _output(out, M, N, out_dtype, inp)
    if workspace is None:
        need = int(lib().dmr_qlinear_bf16_fused_workspace_bytes(M, K, N, pro, 1 if residual is not None else 0))
        if need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=inp.device)    # device memory only
    pws, wbytes = _workspace(workspace)
    _check(lib().dmr_qlinear_bf16_forward_fused(pw_, pro, pi, pg, float(eps), pr, M, K, N, po, _out_code(out.dtype),
                                                pws, wbytes, _stream(stream)), "dmr_qlinear_bf16_forward_fused")
    return out


# ---- paged attention -----------------------------------------------------------------------------

_I32 = (torch.int32,)


def _refuse(dev: int, *tensors):
    """Which of (name, tensor, dtypes) a call cannot take.  The calls below look at up to ten tensors and launch kernels of 3 us, so they
    look in one expression, 0.15 us a tensor, and come here only if something is wrong."""
    for name, t, dtypes in tensors:
        if t is not None:
            _dev(t, name, dtypes)
            if t.get_device() != dev:
                raise ValueError(f"{name} must be on the current device")
    raise ValueError("a tensor of this call cannot be used")


def _for(stream):
    """Where a call on ``stream`` makes its own tensors: they are filled, and later reused, in that stream's order."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))


class KvCache:
    """One layer's keys and values in pages: the pools of ``dmr_kv_cache_t``, bf16 or float8_e4m3fn (16-byte pieces of ``pc``
    elements), k ``[pages][kv_heads][page_tokens / 16][head_dim / pc][16][pc]``, v ``[pages][kv_heads][page_tokens / 16][16 / pc][head_dim][pc]``."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: float = 1.0, v_scale: float = 1.0):
        types = (torch.bfloat16, torch.float8_e4m3fn)
        pk, pv = _dev(k, "k", types), _dev(v, "v", types)
        if k.dtype != v.dtype or k.device != v.device:
            raise ValueError("k and v must have one dtype and one device")
        pc = 16 // k.element_size()
        if k.dim() != 6 or tuple(k.shape[4:]) != (16, pc):
            raise ValueError("k must be [pages][kv_heads][page_tokens / 16][head_dim / %d][16][%d]" % (pc, pc))
        pages, heads, blocks, pieces = k.shape[:4]
        if tuple(v.shape) != (pages, heads, blocks, 16 // pc, pieces * pc, pc):
            raise ValueError("v must be [pages][kv_heads][page_tokens / 16][%d][head_dim][%d]" % (16 // pc, pc))
        self.k, self.v, self.device = k, v, k.get_device()
        self.pages, self.page_tokens, self.kv_heads, self.head_dim = pages, 16 * blocks, heads, pieces * pc
        self.k_scale, self.v_scale = float(k_scale), float(v_scale)
        kind = DMR_KV_BF16 if k.dtype == torch.bfloat16 else DMR_KV_E4M3
        self._struct = _KvCacheStruct(pk, pv, pages, self.page_tokens, heads, self.head_dim, kind, self.k_scale, self.v_scale)
        self._ref = ctypes.byref(self._struct)

    @classmethod
    def empty(cls, pages: int, page_tokens: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, k_scale: float = 1.0,
              v_scale: float = 1.0, device="cuda") -> "KvCache":
        """A cache on uninitialised pools of its own."""
        if dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise TypeError("a cache is torch.bfloat16 or torch.float8_e4m3fn")
        pc = 8 if dtype == torch.bfloat16 else 16
        if dmr_kv_page_bytes(page_tokens, kv_heads, head_dim, DMR_KV_BF16 if pc == 8 else DMR_KV_E4M3) == 0:
            raise ValueError("page_tokens, kv_heads or head_dim not supported")
        head = (pages, kv_heads, page_tokens // 16)
        return cls(torch.empty(head + (head_dim // pc, 16, pc), dtype=dtype, device=device),
                   torch.empty(head + (16 // pc, head_dim, pc), dtype=dtype, device=device), k_scale, v_scale)


def dmr_kv_page_bytes(page_tokens: int, kv_heads: int, head_dim: int, kind: int) -> int:
    return int(lib().dmr_kv_page_bytes(page_tokens, kv_heads, head_dim, kind))


def dmr_kv_assign(new_tokens: torch.Tensor, lens: torch.Tensor, free_pages: torch.Tensor, free_count: torch.Tensor,
                  block_table: torch.Tensor, page_tokens: int, rows: int, out=None, stream=None):
    """(query_start, kv_lens, positions, slots, left), all int32; ``block_table`` gets the new pages.  ``out``: the five tensors to
    write; its kv_lens may be ``lens``, and its left may share its first word with ``free_count``."""
    dev = torch._C._cuda_getDevice()
    n, (requests, width) = new_tokens.numel(), block_table.shape
    if requests != n or lens.numel() != n or free_count.numel() < 1:
        raise ValueError("lens must hold a value per request, block_table be [requests][width], free_count hold one value")
    if rows < 0:
        raise ValueError("rows must not be negative")
    if out is None:
        with _for(stream):
            out = tuple(torch.empty(m, dtype=torch.int32, device=lens.device) for m in (n + 1, n, rows, rows, 2))
    start, kv_lens, positions, slots, left = out
    if start.numel() != n + 1 or kv_lens.numel() != n or positions.numel() != rows or slots.numel() != rows or left.numel() != 2:
        raise ValueError("out must be query_start [requests + 1], kv_lens [requests], positions [rows], slots [rows], left [2]")
    i32 = torch.int32
    if not (new_tokens.dtype is i32 and new_tokens.is_contiguous() and new_tokens.get_device() == dev
            and lens.dtype is i32 and lens.is_contiguous() and lens.get_device() == dev
            and free_pages.dtype is i32 and free_pages.is_contiguous() and free_pages.get_device() == dev
            and free_count.dtype is i32 and free_count.is_contiguous() and free_count.get_device() == dev
            and block_table.dtype is i32 and block_table.is_contiguous() and block_table.get_device() == dev
            and start.dtype is i32 and start.is_contiguous() and start.get_device() == dev
            and kv_lens.dtype is i32 and kv_lens.is_contiguous() and kv_lens.get_device() == dev
            and positions.dtype is i32 and positions.is_contiguous() and positions.get_device() == dev
            and slots.dtype is i32 and slots.is_contiguous() and slots.get_device() == dev
            and left.dtype is i32 and left.is_contiguous() and left.get_device() == dev):
        _refuse(dev, ("new_tokens", new_tokens, _I32), ("lens", lens, _I32), ("free_pages", free_pages, _I32), ("free_count", free_count, _I32),
                ("block_table", block_table, _I32), ("query_start", start, _I32), ("kv_lens", kv_lens, _I32), ("positions", positions, _I32),
                ("slots", slots, _I32), ("left", left, _I32))
    status = lib().dmr_kv_assign(n, rows, width, page_tokens, free_pages.numel(), new_tokens.data_ptr(), lens.data_ptr(),
                                 free_pages.data_ptr(), free_count.data_ptr(), block_table.data_ptr(), start.data_ptr(), kv_lens.data_ptr(),
                                 positions.data_ptr(), slots.data_ptr(), left.data_ptr(),
                                 torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream))
    if status:
        raise DmrError(status, "dmr_kv_assign")
    return tuple(out)


def dmr_kv_append(cache: KvCache, qkv: torch.Tensor, q_heads: int, positions: torch.Tensor | None, slots: torch.Tensor,
                  gamma_q: torch.Tensor | None = None, gamma_k: torch.Tensor | None = None, eps: float = 0.0,
                  inv_freq: torch.Tensor | None = None, interleaved: bool = False, out: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
    """qkv [rows][(q_heads + 2 kv_heads) head_dim] to queries [rows][q_heads head_dim] (returned) and to the cache's slots."""
    dev = torch._C._cuda_getDevice()
    D = cache.head_dim
    rows, width = qkv.shape
    if width != (q_heads + 2 * cache.kv_heads) * D:
        raise ValueError("qkv must be [rows][(q_heads + 2 kv_heads) head_dim]")
    if slots.numel() != rows or (positions is not None and positions.numel() != rows):
        raise ValueError("positions and slots must hold one value per row")
    if cache.device != dev:
        raise ValueError("the cache must be on the current device")
    if out is None:
        with _for(stream):
            out = torch.empty((rows, q_heads * D), dtype=torch.bfloat16, device=qkv.device)
    elif out.shape != (rows, q_heads * D):
        raise ValueError("out must be [rows][q_heads head_dim]")
    f32, i32 = torch.float32, torch.int32
    if not (qkv.dtype in _BF16 and qkv.is_contiguous() and qkv.get_device() == dev
            and out.dtype in _BF16 and out.is_contiguous() and out.get_device() == dev
            and slots.dtype is i32 and slots.is_contiguous() and slots.get_device() == dev
            and (positions is None or (positions.dtype is i32 and positions.is_contiguous() and positions.get_device() == dev))
            and (gamma_q is None or (gamma_q.dtype in _BF16 and gamma_q.is_contiguous() and gamma_q.get_device() == dev))
            and (gamma_k is None or (gamma_k.dtype in _BF16 and gamma_k.is_contiguous() and gamma_k.get_device() == dev))
            and (inv_freq is None or (inv_freq.dtype is f32 and inv_freq.is_contiguous() and inv_freq.get_device() == dev))):
        _refuse(dev, ("qkv", qkv, _BF16), ("out", out, _BF16), ("slots", slots, _I32), ("positions", positions, _I32),
                ("gamma_q", gamma_q, _BF16), ("gamma_k", gamma_k, _BF16), ("inv_freq", inv_freq, (f32,)))
    if (gamma_q is not None and gamma_q.shape != (D,)) or (gamma_k is not None and gamma_k.shape != (D,)):
        raise ValueError("gamma_q and gamma_k must be [head_dim]")
    if inv_freq is not None and inv_freq.shape != (D // 2,):
        raise ValueError("inv_freq must be [head_dim / 2]")
    status = lib().dmr_kv_append(cache._ref, qkv.data_ptr(), rows, q_heads, None if gamma_q is None else gamma_q.data_ptr(),
                                 None if gamma_k is None else gamma_k.data_ptr(), eps, None if inv_freq is None else inv_freq.data_ptr(),
                                 DMR_ROPE_ADJACENT if interleaved else DMR_ROPE_HALVES, None if positions is None else positions.data_ptr(),
                                 slots.data_ptr(), out.data_ptr(), torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream))
    if status:
        raise DmrError(status, "dmr_kv_append")
    return out


def dmr_attn_paged_workspace_bytes(rows: int, requests: int, q_heads: int, kv_heads: int, head_dim: int, max_query: int) -> int:
    return int(lib().dmr_attn_paged_workspace_bytes(rows, requests, q_heads, kv_heads, head_dim, max_query))


def dmr_attn_paged(cache: KvCache, q: torch.Tensor, q_heads: int, query_start: torch.Tensor, kv_lens: torch.Tensor,
                   block_table: torch.Tensor, max_query: int, scale: float, out: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Causal attention of rows q [rows][q_heads head_dim] over their requests' keys in the cache.  A new ``out`` is zeroed, since
    rows of no request are not written; a given one is apart from ``q``.  Single tokens on long histories beside a chunk are better
    served by a call of their own with ``max_query`` 1."""
    dev = torch._C._cuda_getDevice()
    n, D = kv_lens.numel(), cache.head_dim
    (rows, width), (requests, columns) = q.shape, block_table.shape
    if width != q_heads * D:
        raise ValueError("q must be [rows][q_heads head_dim]")
    if query_start.numel() != n + 1 or requests != n:
        raise ValueError("query_start must be [requests + 1], block_table [requests][width]")
    if cache.device != dev:
        raise ValueError("the cache must be on the current device")
    if out is None:
        with _for(stream):
            out = torch.zeros((rows, width), dtype=torch.bfloat16, device=q.device)
    elif out.shape != (rows, width):
        raise ValueError("out must be [rows][q_heads head_dim]")
    i32 = torch.int32
    if not (q.dtype in _BF16 and q.is_contiguous() and q.get_device() == dev
            and out.dtype in _BF16 and out.is_contiguous() and out.get_device() == dev
            and query_start.dtype is i32 and query_start.is_contiguous() and query_start.get_device() == dev
            and kv_lens.dtype is i32 and kv_lens.is_contiguous() and kv_lens.get_device() == dev
            and block_table.dtype is i32 and block_table.is_contiguous() and block_table.get_device() == dev
            and (workspace is None or (workspace.dtype is torch.uint8 and workspace.is_contiguous() and workspace.get_device() == dev))):
        _refuse(dev, ("q", q, _BF16), ("out", out, _BF16), ("query_start", query_start, _I32), ("kv_lens", kv_lens, _I32),
                ("block_table", block_table, _I32), ("workspace", workspace, (torch.uint8,)))
    if workspace is None:
        need = dmr_attn_paged_workspace_bytes(rows, n, q_heads, cache.kv_heads, D, max_query)
        if need > 0:
            with _for(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)    # device memory only
    status = lib().dmr_attn_paged(cache._ref, q.data_ptr(), rows, q_heads, n, query_start.data_ptr(), kv_lens.data_ptr(), block_table.data_ptr(),
                                  columns, max_query, scale, out.data_ptr(), None if workspace is None else workspace.data_ptr(),
                                  0 if workspace is None else workspace.numel(),
                                  torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream))
    if status:
        raise DmrError(status, "dmr_attn_paged")
    return out
