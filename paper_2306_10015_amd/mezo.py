"""Python binding of libmezo (include/mezo.h): argument marshalling only.

Every step of the engine runs in the library's HIP kernels; PyTorch supplies
device memory and the current stream. Importing this module loads
``libmezo.so`` from this directory and raises if it is not built (build it
with ``python -m paper_2306_10015_amd.build``); there is no fallback.

    from paper_2306_10015_amd import mezo
    params = [torch.randn(1024, 1024, device="cuda") * 0.02 for _ in range(4)]
    ps = mezo.ParamSet(params)                       # tensor_id = position
    s = (machine_id, step, sample)
    ps.perturb(s, +eps); ...; ps.perturb(s, -2 * eps); ...; ps.perturb(s, +eps)
    q = mezo.quantize_projgrad([(l_plus - l_minus) / (2 * eps)])
    ps.update_multi(seeds, q_all, lr=eta / n_grads)  # Algorithm 1 apply loop
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import struct
from pathlib import Path
from typing import Iterable, Sequence

import numpy as np
import torch

LIB_PATH = Path(__file__).resolve().parent / "libmezo.so"

OK, EINVAL, EDTYPE, EOVERLAP, EORDER, ERANGE, EHIP, ENOMEM = 0, -1, -2, -3, -4, -5, -6, -7
F32, BF16, NF4 = 0, 1, 2
#: NF4 elements per absmax value.
NF4_BLOCK = 64
#: 8-bit storage: elements of a row that share a scale.
F8_BLOCK = 128
GAUSS_FAST, GAUSS_PORTABLE = 0, 1
LINEAR, SIGNED_LOG = 0, 1
#: Signed-log slope of a base-2 log: code 127 decodes just inside fp32.
LOG2_ALPHA = 1.0 / math.log(2.0)
MAX_NUMEL = 1 << 34

#: Layout of mezo_seed_t: (machine u64, step u32, sample u32), 16 bytes.
SEED_DTYPE = np.dtype([("machine", "<u8"), ("step", "<u4"), ("sample", "<u4")])


class Seed(ctypes.Structure):
    _fields_ = [("machine", ctypes.c_uint64), ("step", ctypes.c_uint32),
                ("sample", ctypes.c_uint32)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("numel", ctypes.c_uint64),
                ("tensor_id", ctypes.c_uint32), ("dtype", ctypes.c_uint32),
                ("absmax", ctypes.c_void_p), ("first", ctypes.c_uint64)]


class Codec(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_uint32), ("scale", ctypes.c_float), ("alpha", ctypes.c_float)]


#: Layout of mezo_attention_t: 7 pointers, 12 u64, 6 u32, 2 floats.
_ATTENTION = struct.Struct("=7Q12Q6I2f")


class Step(ctypes.Structure):
    _fields_ = [("seeds", ctypes.c_void_p), ("q", ctypes.c_void_p), ("K", ctypes.c_uint32),
                ("lr", ctypes.c_float)]


#: Every symbol include/mezo.h declares.
EXPORTS = ("mezo_paramset_create", "mezo_paramset_destroy", "mezo_paramset_numel",
           "mezo_paramset_set_gaussian",
           "mezo_perturb", "mezo_perturb_multi", "mezo_update_multi", "mezo_replay", "mezo_replay_noalloc",
           "mezo_perturb_from",
           "mezo_update_multi_from", "mezo_checksum", "quantize_projgrad",
           "mezo_dequantize", "mezo_nf4_quantize", "mezo_nf4_dequantize",
           "mezo_f8_quantize", "mezo_f8_matmul_workspace", "mezo_f8_matmul",
           "mezo_f8_linear_workspace", "mezo_f8_linear",
           "mezo_attention_workspace", "mezo_attention",
           "mezo_token_loss_workspace", "mezo_token_loss", "mezo_debug_generate", "mezo_debug_box_muller",
           "mezo_strerror", "mezo_last_error", "mezo_version")


def _load() -> ctypes.CDLL:
    # libmezo must run on the same HIP runtime as torch: the streams and device
    # pointers it receives belong to that runtime. torch carries its own copy
    # (same SONAME); importing torch first (above) makes the dynamic loader bind
    # libmezo to it instead of loading a second runtime.
    if not LIB_PATH.exists():
        raise ImportError(f"{LIB_PATH} is not built: run python -m paper_2306_10015_amd.build")
    L = ctypes.CDLL(str(LIB_PATH))
    vp, u32, u64, i32, f32 = (ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int,
                               ctypes.c_float)
    L.mezo_paramset_create.argtypes = [ctypes.POINTER(Tensor), u32, ctypes.POINTER(vp)]
    L.mezo_paramset_create.restype = i32
    L.mezo_paramset_destroy.argtypes = [vp]
    L.mezo_paramset_destroy.restype = None
    L.mezo_paramset_numel.argtypes = [vp]
    L.mezo_paramset_numel.restype = u64
    L.mezo_paramset_set_gaussian.argtypes = [vp, u32]
    L.mezo_paramset_set_gaussian.restype = i32
    L.mezo_perturb.argtypes = [vp, Seed, f32, vp]
    L.mezo_perturb.restype = i32
    L.mezo_perturb_multi.argtypes = [vp, vp, vp, u32, vp]
    L.mezo_perturb_multi.restype = i32
    L.mezo_update_multi.argtypes = [vp, vp, vp, u32, ctypes.POINTER(Codec), f32, vp]
    L.mezo_update_multi.restype = i32
    L.mezo_replay.argtypes = [vp, ctypes.POINTER(Step), u32, ctypes.POINTER(Codec), vp]
    L.mezo_replay.restype = i32
    L.mezo_replay_noalloc.argtypes = [vp, ctypes.POINTER(Step), u32, ctypes.POINTER(Codec), vp]
    L.mezo_replay_noalloc.restype = i32
    L.mezo_perturb_from.argtypes = [vp, vp, Seed, f32, vp]
    L.mezo_perturb_from.restype = i32
    L.mezo_update_multi_from.argtypes = [vp, vp, vp, vp, u32, ctypes.POINTER(Codec), f32, vp]
    L.mezo_update_multi_from.restype = i32
    L.mezo_checksum.argtypes = [vp, vp, vp]
    L.mezo_checksum.restype = i32
    L.quantize_projgrad.argtypes = [vp, vp, u32, ctypes.POINTER(Codec)]
    L.quantize_projgrad.restype = i32
    L.mezo_dequantize.argtypes = [vp, vp, u32, ctypes.POINTER(Codec)]
    L.mezo_dequantize.restype = i32
    L.mezo_nf4_quantize.argtypes = [vp, u32, u64, vp, vp, vp]
    L.mezo_nf4_quantize.restype = i32
    L.mezo_nf4_dequantize.argtypes = [vp, vp, u64, vp, u32, vp]
    L.mezo_nf4_dequantize.restype = i32
    L.mezo_f8_quantize.argtypes = [vp, u32, u64, u64, u64, vp, vp, vp]
    L.mezo_f8_quantize.restype = i32
    L.mezo_f8_matmul_workspace.argtypes = [u64, u64, u64, u32]
    L.mezo_f8_matmul_workspace.restype = u64
    L.mezo_f8_matmul.argtypes = [vp, vp, vp, vp, u64, u64, u64, vp, u32, u64, vp, u64, vp]
    L.mezo_f8_matmul.restype = i32
    L.mezo_f8_linear_workspace.argtypes = [u64, u64, u64, u32]
    L.mezo_f8_linear_workspace.restype = u64
    L.mezo_f8_linear.argtypes = [vp, u32, u64, vp, vp, u64, u64, u64, vp, u32, u64, vp, u64, vp]
    L.mezo_f8_linear.restype = i32
    L.mezo_attention_workspace.argtypes = [vp]
    L.mezo_attention_workspace.restype = u64
    L.mezo_attention.argtypes = [vp, vp, u64, vp]
    L.mezo_attention.restype = i32
    L.mezo_token_loss_workspace.argtypes = [u64, u64]
    L.mezo_token_loss_workspace.restype = u64
    L.mezo_token_loss.argtypes = [vp, u32, u64, u64, u64, vp, vp, vp, vp, u64, vp]
    L.mezo_token_loss.restype = i32
    L.mezo_debug_generate.argtypes = [Seed, u32, u64, u64, u32, vp, vp, vp]
    L.mezo_debug_generate.restype = i32
    L.mezo_debug_box_muller.argtypes = [vp, u64, u32, vp, vp]
    L.mezo_debug_box_muller.restype = i32
    L.mezo_strerror.argtypes = [i32]
    L.mezo_strerror.restype = ctypes.c_char_p
    L.mezo_last_error.argtypes = []
    L.mezo_last_error.restype = ctypes.c_char_p
    L.mezo_version.argtypes = []
    L.mezo_version.restype = i32
    return L


lib = _load()


class MezoError(RuntimeError):
    def __init__(self, code: int, what: str):
        msg = lib.mezo_strerror(code).decode()
        if code in (EHIP, ENOMEM):
            msg += f" ({lib.mezo_last_error().decode()})"
        super().__init__(f"{what}: {msg} [code {code}]")
        self.code = code


def _check(rc: int, what: str) -> None:
    if rc != OK:
        raise MezoError(rc, what)


def codec(kind: int = LINEAR, scale: float = 1.0 / 127.0, alpha: float = LOG2_ALPHA) -> Codec:
    return Codec(kind, scale, alpha)


DEFAULT_CODEC = codec()


def _seed(s) -> Seed:
    if isinstance(s, Seed):
        return s
    if isinstance(s, np.void):
        return Seed(int(s["machine"]), int(s["step"]), int(s["sample"]))
    m, t, j = s
    return Seed(int(m), int(t), int(j))


def seeds_array(seeds) -> np.ndarray:
    """Any sequence of (machine, step, sample) -> contiguous SEED_DTYPE array."""
    if isinstance(seeds, np.ndarray) and seeds.dtype == SEED_DTYPE:
        return np.ascontiguousarray(seeds)
    out = np.zeros(len(seeds), dtype=SEED_DTYPE)
    for i, s in enumerate(seeds):
        out[i] = s if isinstance(s, np.void) else (int(s[0]), int(s[1]), int(s[2]))
    return out


def _stream_ptr(stream) -> int | None:
    if stream is None:
        # (torch.cuda.current_stream() makes a Stream object: 3 us)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _dtype_code(t) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported parameter dtype {t.dtype}")


class NF4Tensor:
    """A tensor of ``numel`` elements in 4-bit NormalFloat storage (the 4-bit
    forward-only variant): ``codes`` (uint8, ceil(numel / 2) bytes, element
    2i in the low nibble of byte i) and ``absmax`` (float32, one per block of
    64 elements), both contiguous device tensors owned by torch."""

    def __init__(self, codes, absmax, numel: int):
        if codes.dtype != torch.uint8 or absmax.dtype != torch.float32:
            raise TypeError("codes must be uint8 and absmax float32")
        if not (codes.is_cuda and absmax.is_cuda and codes.is_contiguous() and absmax.is_contiguous()):
            raise ValueError("codes and absmax must be contiguous CUDA tensors")
        if codes.numel() < (numel + 1) // 2 or absmax.numel() < (numel + NF4_BLOCK - 1) // NF4_BLOCK:
            raise ValueError("codes / absmax too small for numel")
        self.codes, self.absmax, self._numel = codes, absmax, int(numel)

    @classmethod
    def empty(cls, numel: int, device="cuda") -> "NF4Tensor":
        return cls(torch.empty((numel + 1) // 2, dtype=torch.uint8, device=device),
                   torch.empty((numel + NF4_BLOCK - 1) // NF4_BLOCK, dtype=torch.float32, device=device),
                   numel)

    def numel(self) -> int:
        return self._numel

    @property
    def device(self):
        return self.codes.device

    @property
    def is_cuda(self) -> bool:
        return True


def nf4_quantize(values, out: NF4Tensor | None = None, stream=None) -> NF4Tensor:
    """values (contiguous fp32/bf16 device tensor) -> NF4 storage."""
    n = values.numel()
    out = NF4Tensor.empty(n, values.device) if out is None else out
    if out.numel() != n or not values.is_contiguous():
        raise ValueError("size mismatch or non-contiguous values")
    with torch.cuda.device(values.device):
        _check(lib.mezo_nf4_quantize(values.data_ptr(), _dtype_code(values), n, out.codes.data_ptr(),
                                     out.absmax.data_ptr(), _stream_ptr(stream)), "mezo_nf4_quantize")
    return out


def nf4_dequantize(t: NF4Tensor, dtype=None, out=None, stream=None):
    """NF4 storage -> a fp32 (default) or bf16 device tensor of numel elements."""
    if out is None:
        out = torch.empty(t.numel(), dtype=dtype or torch.float32, device=t.device)
    if out.numel() != t.numel() or not out.is_contiguous():
        raise ValueError("size mismatch or non-contiguous out")
    with torch.cuda.device(t.device):
        _check(lib.mezo_nf4_dequantize(t.codes.data_ptr(), t.absmax.data_ptr(), t.numel(), out.data_ptr(),
                                       _dtype_code(out), _stream_ptr(stream)), "mezo_nf4_dequantize")
    return out


# ---- the forward pass ------------------------------------------------------
#
# None of these operators has a backward pass. They may be called on tensors that
# require a gradient (a model's parameters do unless told otherwise); a backward
# pass through their outputs raises.

_NO_SWITCH = contextlib.nullcontext()
_DEVICES = 0


def _on(device, stream):
    """Run a call on `device`, its outputs and scratch allocated on the stream
    it runs on (memory of another stream's pool could still be in use there)."""
    global _DEVICES
    if not _DEVICES:
        _DEVICES = torch.cuda.device_count()
    if stream is None and _DEVICES == 1:
        return _NO_SWITCH  # (a context of its own costs a small call 2 us)
    stack = contextlib.ExitStack()
    stack.enter_context(torch.cuda.device(device))
    if stream is not None:
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        stack.enter_context(torch.cuda.stream(stream))
    return stack


def _rows_of(t, what: str):
    """A 2-D CUDA tensor whose rows are contiguous, and the elements between them."""
    shape = t.shape
    if len(shape) != 2 or not t.is_cuda:
        raise ValueError(f"{what}: a 2-D CUDA tensor")
    rows, cols = shape
    if rows == 0 or cols == 0:
        raise ValueError(f"{what}: empty")
    ld, step = t.stride()
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    return rows, cols, ld if rows > 1 else cols


def _same_device(first, *others):
    """All on the device of `first`, a CUDA tensor (with one device: all on it)."""
    if _DEVICES == 1:
        for t in others:
            if t is not None and not t.is_cuda:
                raise ValueError(f"tensors on several devices: {first.device} and {t.device}")
        return
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"tensors on several devices: {first.device} and {t.device}")


def _scratch(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _ptr(t):
    return None if t is None else t.data_ptr()


class _NoBackward(torch.autograd.Function):
    """Stands for an operator in autograd's graph: differentiating through it is
    an error, not a gradient left out."""

    @staticmethod
    def forward(ctx, name, count, *tensors):
        ctx.name = name
        ctx.mark_dirty(*tensors[:count])  # (the operator wrote them)
        return tensors[:count]

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(f"mezo.{ctx.name} has no backward pass (the method takes no derivative): "
                           "call it under torch.no_grad(), or on detached tensors")


def _no_backward(name, outputs, *inputs):
    """Outputs of inputs that require a gradient require one too."""
    if any(t is not None and t.requires_grad for t in inputs) and torch.is_grad_enabled():
        _NoBackward.apply(name, len(outputs), *outputs, *inputs)


class F8Matrix:
    """A [rows, cols] matrix in 8-bit storage: ``codes`` (uint8, [rows, B * 128]
    with B = ceil(cols / 128) blocks a row, e4m3, zeros after the last column)
    and ``scales`` (uint8, [rows, B rounded up to a multiple of 4], a block's
    scale 2^(byte - 127)), both contiguous device tensors owned by torch."""

    def __init__(self, codes, scales, rows: int, cols: int):
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
            raise TypeError("codes and scales must be uint8")
        rows, cols = int(rows), int(cols)
        blocks = (cols + F8_BLOCK - 1) // F8_BLOCK
        if rows < 1 or cols < 1 or codes.shape != (rows, blocks * F8_BLOCK) \
                or scales.shape != (rows, (blocks + 3) // 4 * 4):
            raise ValueError("codes / scales do not have the sizes of a [rows, cols] matrix")
        if not (codes.is_cuda and scales.is_cuda and codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales must be contiguous CUDA tensors")
        _same_device(codes, scales)
        self.codes, self.scales, self.rows, self.cols = codes, scales, rows, cols

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "F8Matrix":
        blocks = (int(cols) + F8_BLOCK - 1) // F8_BLOCK
        return cls(torch.empty(rows, blocks * F8_BLOCK, dtype=torch.uint8, device=device),
                   torch.empty(rows, (blocks + 3) // 4 * 4, dtype=torch.uint8, device=device), rows, cols)

    @property
    def shape(self):
        return self.rows, self.cols

    @property
    def device(self):
        return self.codes.device


def f8_quantize(values, out: F8Matrix | None = None, stream=None) -> F8Matrix:
    """values (fp32/bf16 [rows, cols], contiguous rows) -> 8-bit storage."""
    rows, cols, ld = _rows_of(values, "values")
    dtype = _dtype_code(values)
    if out is not None and out.shape != (rows, cols):
        raise ValueError(f"out is {out.shape}, values {(rows, cols)}")
    with _on(values.device, stream):
        out = F8Matrix.empty(rows, cols, values.device) if out is None else out
        _same_device(values, out.codes)
        _check(lib.mezo_f8_quantize(values.data_ptr(), dtype, rows, cols, ld, out.codes.data_ptr(),
                                    out.scales.data_ptr(), _stream_ptr(None)), "mezo_f8_quantize")
    return out


def f8_matmul(x: F8Matrix, w: F8Matrix, dtype=None, out=None, stream=None):
    """x w^T of two 8-bit matrices, [m, k] and [n, k], as a [m, n] tensor of
    dtype (torch.bfloat16, the default, or torch.float32: see mezo_f8_matmul)."""
    if x.cols != w.cols:
        raise ValueError(f"x has {x.cols} columns, w {w.cols}")
    m, n, k = x.rows, w.rows, x.cols
    with _on(x.device, stream):
        if out is None:
            out = torch.empty(m, n, dtype=dtype or torch.bfloat16, device=x.device)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype {dtype}")
        if out.shape != (m, n):
            raise ValueError(f"out is {tuple(out.shape)}, the product {(m, n)}")
        _same_device(x.codes, w.codes, out)
        code, ldc = _dtype_code(out), _rows_of(out, "out")[2]
        nbytes = lib.mezo_f8_matmul_workspace(m, n, k, code)
        ws = _scratch(nbytes, x.device)
        _check(lib.mezo_f8_matmul(x.codes.data_ptr(), x.scales.data_ptr(), w.codes.data_ptr(), w.scales.data_ptr(),
                                  m, n, k, out.data_ptr(), code, ldc, _ptr(ws), nbytes, _stream_ptr(None)),
               "mezo_f8_matmul")
    return out


def f8_linear(x, w: F8Matrix, dtype=None, out=None, stream=None):
    """A layer's product: the activations x (fp32/bf16 [m, k]) quantized, times
    the weights w ([n, k]) in 8-bit storage: [m, n] of dtype (x's by default).
    The same as f8_matmul(f8_quantize(x), w, dtype), in one call."""
    m, k, ldx = _rows_of(x, "x")
    if k != w.cols:
        raise ValueError(f"x has {k} columns, w {w.cols}")
    n, x_code = w.rows, _dtype_code(x)
    with _on(x.device, stream):
        if out is None:
            out = torch.empty(m, n, dtype=dtype or x.dtype, device=x.device)
            ldc = n
        else:
            if dtype is not None and out.dtype != dtype:
                raise TypeError(f"out is {out.dtype}, dtype {dtype}")
            if out.shape != (m, n):
                raise ValueError(f"out is {tuple(out.shape)}, the product {(m, n)}")
            ldc = _rows_of(out, "out")[2]
        _same_device(x, w.codes, out)
        code = _dtype_code(out)
        nbytes = lib.mezo_f8_linear_workspace(m, n, k, code)
        ws = _scratch(nbytes, x.device)
        _check(lib.mezo_f8_linear(x.data_ptr(), x_code, ldx, w.codes.data_ptr(), w.scales.data_ptr(), m, n, k,
                                  out.data_ptr(), code, ldc, _ptr(ws), nbytes, _stream_ptr(None)), "mezo_f8_linear")
    if x.requires_grad:
        _no_backward("f8_linear", (out,), x)
    return out


class Documents:
    """The documents of an attention call: ``table``, a device tensor int64
    [documents, 5] of (q_first, q_len, k_first, k_len, prefix) as in mezo.h, and
    the most queries and keys a document has. Use ``Documents.of`` to make one
    from lengths, checked. ``covered``: the documents' queries are tokens 0 ..
    covered - 1, each of one document (None: not known)."""

    def __init__(self, table, max_q: int, max_k: int, covered: int | None = None):
        if table.dtype != torch.int64:
            raise TypeError(f"table must be int64, got {table.dtype}")
        shape = table.shape
        if len(shape) != 2 or shape[1] != 5 or not table.is_cuda or not table.is_contiguous():
            raise ValueError("table: a contiguous CUDA tensor [documents, 5]")
        if max_q < 0 or max_k < 0:
            raise ValueError("max_q and max_k must not be negative")
        self.table, self.count, self.max_q, self.max_k = table, shape[0], int(max_q), int(max_k)
        self.covered = covered

    @classmethod
    def of(cls, q_lens, k_lens=None, prefix=None, q_first=None, k_first=None, device="cuda") -> "Documents":
        """From sequences of lengths: q_lens queries and k_lens keys a document
        (q_lens by default), the visible prefix (0), and where each begins
        (packed one after another by default)."""

        def ints(x, default):
            out = [int(v) for v in (default if x is None else x)]
            if len(out) != len(q_lens) or any(v < 0 for v in out):
                raise ValueError("one value that is not negative for each document")
            return out

        def packed(lens):
            at, out = 0, []
            for n in lens:
                out.append(at)
                at += n
            return out

        q_lens = list(q_lens)
        q_lens = ints(q_lens, q_lens)
        k_lens = ints(k_lens, q_lens)
        q_first, k_first = ints(q_first, packed(q_lens)), ints(k_first, packed(k_lens))
        spans = sorted((a, a + n) for a, n in zip(q_first, q_lens) if n)
        if any(b > c for (_, b), (c, _) in zip(spans, spans[1:])):
            raise ValueError("the documents' queries overlap")
        rows = list(zip(q_first, q_lens, k_first, k_lens, ints(prefix, [0] * len(q_lens))))
        table = torch.tensor(rows, dtype=torch.int64, device=device).reshape(len(rows), 5)
        gaps = sum(q_lens) != max((b for _, b in spans), default=0)
        return cls(table, max(q_lens, default=0), max(k_lens, default=0), 0 if gaps else sum(q_lens))


def _heads_of(t, what: str):
    """(tokens, heads, dim) of a 3-D CUDA tensor with contiguous heads, and the
    elements from one token and from one head to the next."""
    shape = t.shape
    if len(shape) != 3 or not t.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor [tokens, heads, dim]")
    tokens, heads, dim = shape
    st, sh, sd = t.stride()
    if dim > 1 and sd != 1:
        raise ValueError(f"{what}: the elements of a head must be contiguous")
    if st < 0 or sh < 0:
        raise ValueError(f"{what}: negative strides")
    return tokens, heads, dim, st if tokens > 1 else heads * dim, sh if heads > 1 else dim


def attention(q, k, v, docs: Documents, causal: bool = True, scale: float | None = None, softcap: float = 0.0,
              slopes=None, out=None, return_lse: bool = False, stream=None):
    """Attention of a batch of documents (mezo_attention): q [tokens, heads,
    dim], k and v [tokens, kv_heads, dim] of fp32 or bf16, each with any token
    and head strides that are multiples of 16 bytes. scale is 1 / sqrt(dim) by
    default; slopes, fp32 [heads], biases scores by -slope * distance. Returns
    out, like q, and with return_lse the pair (out, lse), lse fp32 [tokens, heads].
    Tokens of no document: 0 and -inf, as of a query that sees no key; but with
    ``out`` given they keep what it holds, and with documents whose ``covered``
    is not known they are not written."""
    tq, heads, dim, q_token, q_head = _heads_of(q, "q")
    tk, kv_heads, k_dim, k_token, k_head = _heads_of(k, "k")
    tv, v_heads, v_dim, v_token, v_head = _heads_of(v, "v")
    if (tk, kv_heads) != (tv, v_heads) or not dim == k_dim == v_dim:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not fit together")
    if kv_heads == 0 or heads % kv_heads:
        raise ValueError(f"{heads} heads over {kv_heads} key/value heads")
    dtype = _dtype_code(q)
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError(f"q, k and v are {q.dtype}, {k.dtype} and {v.dtype}")
    if slopes is not None and (slopes.dtype != torch.float32 or slopes.shape != (heads,) or not slopes.is_contiguous()):
        raise ValueError(f"slopes: a contiguous float32 tensor of {heads}")
    with _on(q.device, stream):
        bare = docs.covered is not None and docs.covered < tq  # some tokens are of no document
        if out is None:
            out = (torch.zeros if bare else torch.empty)((tq, heads, dim), dtype=q.dtype, device=q.device)
            o_token, o_head = heads * dim, dim
        else:
            if out.dtype != q.dtype or out.shape != q.shape:
                raise ValueError("out must be like q")
            _, _, _, o_token, o_head = _heads_of(out, "out")
        _same_device(q, k, v, out, slopes, docs.table)
        lse = torch.empty((tq, heads), dtype=torch.float32, device=q.device) if return_lse else None
        if bare and return_lse:
            lse.fill_(-math.inf)
        a = _ATTENTION.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _ptr(lse) or 0,
                            docs.table.data_ptr(), _ptr(slopes) or 0, tq, tk, q_token, q_head, k_token, k_head,
                            v_token, v_head, o_token, o_head, docs.max_q, docs.max_k, docs.count, heads,
                            kv_heads, dim, dtype, 1 if causal else 0,
                            1.0 / math.sqrt(dim) if scale is None else scale, softcap)
        nbytes = lib.mezo_attention_workspace(a)
        ws = _scratch(nbytes, q.device)
        _check(lib.mezo_attention(a, _ptr(ws), nbytes, _stream_ptr(None)), "mezo_attention")
    if q.requires_grad or k.requires_grad or v.requires_grad or (slopes is not None and slopes.requires_grad):
        _no_backward("attention", (out, lse) if return_lse else (out,), q, k, v, slopes)
    return (out, lse) if return_lse else out


def token_loss(logits, targets, stream=None):
    """The cross entropy of each token and the mean over those that count:
    logits fp32/bf16 [tokens, vocabulary] with contiguous rows, targets int64
    [tokens], negative where a token does not count. Returns (losses, mean),
    fp32 device tensors of [tokens] and of no dimension."""
    rows, vocab, ld = _rows_of(logits, "logits")
    dtype = _dtype_code(logits)
    if targets.dtype != torch.int64:
        raise TypeError(f"targets must be int64, got {targets.dtype}")
    if targets.shape != (rows,) or not targets.is_contiguous():
        raise ValueError(f"targets: a contiguous tensor of {rows}")
    _same_device(logits, targets)
    with _on(logits.device, stream):
        losses = torch.empty(rows, dtype=torch.float32, device=logits.device)
        mean = torch.empty((), dtype=torch.float32, device=logits.device)
        nbytes = lib.mezo_token_loss_workspace(rows, vocab)
        ws = _scratch(nbytes, logits.device)
        _check(lib.mezo_token_loss(logits.data_ptr(), dtype, rows, vocab, ld, targets.data_ptr(), losses.data_ptr(),
                                   mean.data_ptr(), _ptr(ws), nbytes, _stream_ptr(None)), "mezo_token_loss")
    if logits.requires_grad:
        _no_backward("token_loss", (losses, mean), logits)
    return losses, mean


def _tensor_struct(t, tid: int, first: int = 0) -> Tensor:
    if isinstance(t, NF4Tensor):
        return Tensor(t.codes.data_ptr(), t.numel(), tid, NF4, t.absmax.data_ptr(), first)
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("parameters must be contiguous CUDA tensors")
    return Tensor(t.data_ptr(), t.numel(), tid, _dtype_code(t), None, first)


class ParamSet:
    """A registered set of parameter tensors (device memory owned by torch):
    fp32 / bf16 torch tensors or NF4Tensor objects.

    ``tensor_ids`` default to the position in ``tensors``; they select each
    tensor's noise stream and must be the same on every machine. ``firsts``
    (default all 0) give, for a shard of a tensor split by element range, the
    index of its first element within the whole tensor (a multiple of 8): the
    shard then computes exactly those elements of the whole tensor.
    """

    def __init__(self, tensors: Sequence, tensor_ids: Iterable[int] | None = None,
                 gaussian: int = GAUSS_FAST, firsts: Iterable[int] | None = None):
        self.tensors = list(tensors)
        devices = set()
        for t in self.tensors:
            devices.add(t.device)
            if isinstance(t, NF4Tensor):
                devices.add(t.absmax.device)
        if len(devices) > 1:
            raise ValueError(f"all tensors of a paramset must live on one device, got {sorted(map(str, devices))}")
        #: the device every call of this paramset runs on (made current for the call)
        self.device = devices.pop() if devices else None
        self._switch = torch.cuda.device_count() > 1
        ids = list(range(len(self.tensors))) if tensor_ids is None else [int(i) for i in tensor_ids]
        if len(ids) != len(self.tensors):
            raise ValueError("one tensor_id per tensor")
        offs = [0] * len(self.tensors) if firsts is None else [int(f) for f in firsts]
        if len(offs) != len(self.tensors):
            raise ValueError("one first-element offset per tensor")
        arr = (Tensor * max(1, len(self.tensors)))()
        for i, (t, tid, f) in enumerate(zip(self.tensors, ids, offs)):
            arr[i] = _tensor_struct(t, tid, f)
        h = ctypes.c_void_p()
        _check(lib.mezo_paramset_create(arr, len(self.tensors), ctypes.byref(h)),
               "mezo_paramset_create")
        self._h = h
        self.tensor_ids = ids
        if gaussian != GAUSS_FAST:
            self.set_gaussian(gaussian)

    def set_gaussian(self, gaussian: int) -> None:
        """GAUSS_FAST (hardware transcendentals) or GAUSS_PORTABLE (binary32
        operations only: bit-identical on any IEEE device)."""
        _check(lib.mezo_paramset_set_gaussian(self._h, int(gaussian)), "mezo_paramset_set_gaussian")

    def _on_device(self):
        """Make the paramset's device current for a call (a stream or pointer
        of another device would not be valid for its kernels); with a single
        visible device there is nothing to switch."""
        return torch.cuda.device(self.device) if self._switch else contextlib.nullcontext()

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    @property
    def numel(self) -> int:
        return int(lib.mezo_paramset_numel(self._h))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            lib.mezo_paramset_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def perturb(self, seed, scale: float, stream=None) -> None:
        """PerturbParameters: theta += scale * z(seed)."""
        with self._on_device():
            _check(lib.mezo_perturb(self._h, _seed(seed), float(scale), _stream_ptr(stream)),
                   "mezo_perturb")

    def perturb_multi(self, seeds, scales, stream=None) -> None:
        """Perturbs in sequence in one pass: theta += scales[i] * z(seeds[i]),
        rounded after each (e.g. restore sample j and perturb for sample j+1)."""
        sa = seeds_array(seeds)
        sc = np.ascontiguousarray(scales, dtype=np.float32)
        if sa.size != sc.size:
            raise ValueError("seeds and scales differ in length")
        with self._on_device():
            _check(lib.mezo_perturb_multi(self._h, sa.ctypes.data, sc.ctypes.data, sa.size, _stream_ptr(stream)),
                   "mezo_perturb_multi")

    def update_multi(self, seeds, q, lr: float, codec_: Codec = DEFAULT_CODEC, stream=None) -> None:
        """Apply loop of one iteration: theta -= lr * sum_k deq(q_k) z(seed_k)."""
        sa = seeds_array(seeds)
        qa = np.ascontiguousarray(q, dtype=np.int8)
        if sa.size != qa.size:
            raise ValueError("seeds and q differ in length")
        with self._on_device():
            _check(lib.mezo_update_multi(self._h, sa.ctypes.data, qa.ctypes.data, sa.size,
                                         ctypes.byref(codec_), float(lr), _stream_ptr(stream)),
                   "mezo_update_multi")

    def perturb_from(self, src: "ParamSet", seed, scale: float, stream=None) -> None:
        """theta = theta_src + scale * z(seed), src unchanged (out of place)."""
        with self._on_device():
            _check(lib.mezo_perturb_from(self._h, src.handle, _seed(seed), float(scale),
                                         _stream_ptr(stream)), "mezo_perturb_from")

    def update_multi_from(self, src: "ParamSet", seeds, q, lr: float,
                          codec_: Codec = DEFAULT_CODEC, stream=None) -> None:
        """theta = theta_src - lr * sum_k deq(q_k) z(seed_k): restore from the
        backup and apply the iteration's gradients in one pass."""
        sa = seeds_array(seeds)
        qa = np.ascontiguousarray(q, dtype=np.int8)
        if sa.size != qa.size:
            raise ValueError("seeds and q differ in length")
        with self._on_device():
            _check(lib.mezo_update_multi_from(self._h, src.handle, sa.ctypes.data, qa.ctypes.data,
                                              sa.size, ctypes.byref(codec_), float(lr),
                                              _stream_ptr(stream)), "mezo_update_multi_from")

    def checksum_into(self, out, stream=None) -> None:
        """Enqueue the 64-bit checksum of every tensor's bits into `out`, a
        device tensor of 8 bytes (ChecksumMatch, Algorithm 1)."""
        if out.numel() * out.element_size() != 8 or not out.is_cuda:
            raise ValueError("out must be an 8-byte device tensor")
        with self._on_device():
            _check(lib.mezo_checksum(self._h, out.data_ptr(), _stream_ptr(stream)), "mezo_checksum")

    def checksum(self, stream=None) -> int:
        """The checksum as a Python int (waits for the stream it ran on)."""
        out = torch.empty(1, dtype=torch.int64, device=self.device)
        self.checksum_into(out, stream)
        if stream is not None:
            # .item() reads on the current stream, which does not wait for `stream`
            if isinstance(stream, torch.cuda.Stream):
                stream.synchronize()
            else:
                torch.cuda.synchronize(self.device)
        return int(out.item()) & 0xFFFFFFFFFFFFFFFF

    def replay(self, steps, codec_: Codec = DEFAULT_CODEC, stream=None) -> None:
        """Late-joiner catch-up: steps = [(seeds, q, lr), ...] in order."""
        self._replay(lib.mezo_replay, "mezo_replay", steps, codec_, stream)

    def replay_noalloc(self, steps, codec_: Codec = DEFAULT_CODEC, stream=None) -> None:
        """replay through mezo_replay_noalloc, the entry point that allocates
        nothing (at most 65536 records; the set must have had a call of
        another engine entry point first)."""
        self._replay(lib.mezo_replay_noalloc, "mezo_replay_noalloc", steps, codec_, stream)

    def _replay(self, fn, what, steps, codec_, stream) -> None:
        keep = []
        arr = (Step * max(1, len(steps)))()
        for i, (s, q, lr) in enumerate(steps):
            sa = seeds_array(s)
            qa = np.ascontiguousarray(q, dtype=np.int8)
            if sa.size != qa.size:
                raise ValueError(f"step {i}: seeds and q differ in length")
            keep.append((sa, qa))
            arr[i] = Step(sa.ctypes.data, qa.ctypes.data, sa.size, float(lr))
        with self._on_device():
            _check(fn(self._h, arr, len(steps), ctypes.byref(codec_), _stream_ptr(stream)), what)


def step_lr(eta: float, n_grads: int, sqrt_scaling: bool = False) -> float:
    """The per-gradient learning rate of one iteration's apply loop: each
    projected gradient is weighted by eta / n_grads (Algorithm 1); with the
    learning rate scaled by the square root of the number of perturbations
    (Section 4) that is eta * sqrt(n) / n = eta / sqrt(n)."""
    if n_grads <= 0:
        raise ValueError("n_grads must be positive")
    return eta / math.sqrt(n_grads) if sqrt_scaling else eta / n_grads


def quantize_projgrad(g, codec_: Codec = DEFAULT_CODEC) -> np.ndarray:
    ga = np.ascontiguousarray(g, dtype=np.float32)
    q = np.zeros(ga.size, dtype=np.int8)
    _check(lib.quantize_projgrad(ga.ctypes.data, q.ctypes.data, ga.size, ctypes.byref(codec_)),
           "quantize_projgrad")
    return q


def dequantize(q, codec_: Codec = DEFAULT_CODEC) -> np.ndarray:
    qa = np.ascontiguousarray(q, dtype=np.int8)
    g = np.zeros(qa.size, dtype=np.float32)
    _check(lib.mezo_dequantize(qa.ctypes.data, g.ctypes.data, qa.size, ctypes.byref(codec_)),
           "mezo_dequantize")
    return g


def debug_generate(seed, tensor_id: int, first: int, count: int, words=True, z=True,
                   stream=None, gaussian: int = GAUSS_FAST):
    """Device tensors (words uint32 as int32 bits, z float32) of elements
    first .. first+count-1 of tensor tensor_id under seed."""
    w = torch.empty(count, dtype=torch.int32, device="cuda") if words else None
    zz = torch.empty(count, dtype=torch.float32, device="cuda") if z else None
    _check(lib.mezo_debug_generate(_seed(seed), int(tensor_id), int(first), int(count),
                                   int(gaussian), None if w is None else w.data_ptr(),
                                   None if zz is None else zz.data_ptr(), _stream_ptr(stream)),
           "mezo_debug_generate")
    return w, zz


def debug_box_muller(words, gaussian: int = GAUSS_FAST, stream=None):
    """z (float32 device tensor) of the given words (int32/uint32-bit device
    tensor, a multiple of 4 long), through the library's Gaussian transform."""
    if words.numel() % 4 or not words.is_contiguous() or words.element_size() != 4:
        raise ValueError("words: contiguous 32-bit device tensor, a multiple of 4 long")
    z = torch.empty(words.numel(), dtype=torch.float32, device=words.device)
    _check(lib.mezo_debug_box_muller(words.data_ptr(), words.numel() // 4, int(gaussian), z.data_ptr(),
                                     _stream_ptr(stream)), "mezo_debug_box_muller")
    return z


def version() -> int:
    return int(lib.mezo_version())
