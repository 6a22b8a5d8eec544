"""Python binding of libsparcml.so (the gfx950 SparCML C ABI, include/sparcml.h).

Argument marshalling only: torch tensors supply device memory and the
current HIP stream; every step of the computation runs in the library's HIP
kernels.  There is no fallback path -- if the library is missing or the
device is not usable, calls raise.

Index tensors are int32 holding the uint32 bit patterns of the ABI.
"""
from __future__ import annotations

import array
import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libsparcml.so")

OK, EINVAL, ECAPACITY, EWORKSPACE, EUNSORTED, EHIP = 0, -1, -2, -3, -4, -5
OP_TOPK, OP_QUANTIZE, OP_REDUCE, OP_DENSIFY, OP_QUANTIZE_BUCKETED, OP_CONCAT, OP_VALIDATE = 1, 2, 3, 4, 5, 6, 7
OP_TENSORS, OP_LOGPROB, OP_POLICY, OP_PREFERENCE = 8, 9, 10, 11
F32, BF16, F16 = 0, 1, 2


class Stream(ctypes.Structure):
    """Mirror of ``sparcml_stream``."""
    _fields_ = [
        ("idx", ctypes.c_void_p),
        ("val", ctypes.c_void_p),
        ("qval", ctypes.c_void_p),
        ("qscale", ctypes.c_void_p),
        ("nnz", ctypes.c_uint64),
        ("is_dense", ctypes.c_uint32),
        ("qbits", ctypes.c_uint32),
    ]


class Tensor(ctypes.Structure):
    """Mirror of ``sparcml_tensor``."""
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [
        ("n", ctypes.c_uint64),
        ("decay", ctypes.c_float),
        ("lr_scale", ctypes.c_float),
    ]


# The same as bytes, for an array of them from their columns.
_TENSOR_COLUMNS = ("param", "grad", "m", "v", "m_scale", "v_scale", "copy", "n", "decay", "lr_scale")
_pack_tensor = struct.Struct("8Q2f").pack


class Tensors(ctypes.Structure):
    """Mirror of ``sparcml_tensors`` (the plan of a model's tensors)."""
    _fields_ = [
        ("ws", ctypes.c_void_p),
        ("total", ctypes.c_uint64),
        ("chunks", ctypes.c_uint64),
        ("count", ctypes.c_uint32),
        ("grad_type", ctypes.c_uint32),
        ("copy_type", ctypes.c_uint32),
        ("state_bits", ctypes.c_uint32),
        ("check", ctypes.c_uint64),
    ]


class AdamwArgs(ctypes.Structure):
    """Mirror of ``sparcml_adamw_args``."""
    _fields_ = [(name, ctypes.c_double) for name in ("lr", "beta1", "beta2", "eps", "grad_scale")] + [
        ("seed", ctypes.c_uint64),
        ("step", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
    ]


class Logits(ctypes.Structure):
    """Mirror of ``sparcml_logits``."""
    _fields_ = [
        ("x", ctypes.c_void_p),
        ("label", ctypes.c_void_p),
        ("rows", ctypes.c_uint64),
        ("vocab", ctypes.c_uint64),
        ("ld", ctypes.c_uint64),
        ("type", ctypes.c_uint32),
        ("scale", ctypes.c_float),
    ]


class PolicyArgs(ctypes.Structure):
    """Mirror of ``sparcml_policy_args``."""
    _fields_ = [(name, ctypes.c_void_p) for name in ("old_logp", "ref_logp", "adv", "weight")] + [
        (name, ctypes.c_float) for name in ("clip_lo", "clip_hi", "kl", "grad_scale")]


class SparcmlError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status}): {last_error()}")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libsparcml.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_1802_08021_amd.build` "
            "(there is no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, u64, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int
    L.sparcml_workspace_size.argtypes = [i32, i32, u64, u64, ctypes.c_double, ctypes.POINTER(ctypes.c_size_t)]
    L.sparcml_workspace_size.restype = i32
    L.sparcml_topk_sparsify.argtypes = [i32, vp, u64, u64, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.sparcml_topk_sparsify.restype = i32
    L.sparcml_topk_bucketed.argtypes = [i32, vp, vp, u64, ctypes.c_float, u64, u64, vp, vp, vp]
    L.sparcml_topk_bucketed.restype = i32
    L.sparcml_topk_bucketed_count.argtypes = [u64, u64, u64]
    L.sparcml_topk_bucketed_count.restype = u64
    L.sparcml_quantize.argtypes = [i32, ctypes.POINTER(Stream), i32, u64, vp, vp, vp, vp,
                                   ctypes.c_size_t, vp]
    L.sparcml_quantize.restype = i32
    L.sparcml_quantize_bucketed.argtypes = [i32, ctypes.POINTER(Stream), i32, u64, u64, vp, vp, vp, vp,
                                            ctypes.c_size_t, vp]
    L.sparcml_quantize_bucketed.restype = i32
    L.sparcml_sparse_reduce.argtypes = [i32, ctypes.POINTER(Stream), u64, ctypes.c_double,
                                        ctypes.POINTER(Stream), vp, vp, vp, ctypes.c_size_t, vp]
    L.sparcml_sparse_reduce.restype = i32
    L.sparcml_sparse_reduce_range.argtypes = [i32, ctypes.POINTER(Stream), u64, u64, u64, ctypes.c_double,
                                              ctypes.POINTER(Stream), vp, vp, vp, ctypes.c_size_t, vp]
    L.sparcml_sparse_reduce_range.restype = i32
    L.sparcml_sparse_reduce_async.argtypes = [i32, ctypes.POINTER(Stream), u64, u64, u64, ctypes.c_double,
                                              ctypes.POINTER(Stream), vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.sparcml_sparse_reduce_async.restype = i32
    L.sparcml_sparse_reduce_async_noalloc.argtypes = [i32, ctypes.POINTER(Stream), u64, u64, u64,
                                                      ctypes.c_double, ctypes.POINTER(Stream), vp, vp, vp, vp]
    L.sparcml_sparse_reduce_async_noalloc.restype = i32
    L.sparcml_concat.argtypes = [i32, ctypes.POINTER(Stream), ctypes.POINTER(u64), u64, ctypes.c_double, u64,
                                 ctypes.POINTER(Stream), vp, ctypes.c_size_t, vp]
    L.sparcml_concat.restype = i32
    L.sparcml_validate_streams.argtypes = [i32, ctypes.POINTER(Stream), u64, u64, vp, ctypes.c_size_t, vp]
    L.sparcml_validate_streams.restype = i32
    L.sparcml_split_bounds.argtypes = [i32, u64, ctypes.POINTER(u64)]
    L.sparcml_split_bounds.restype = i32
    L.sparcml_densify.argtypes = [ctypes.POINTER(Stream), u64, vp, vp]
    L.sparcml_densify.restype = i32
    f32 = ctypes.c_float
    L.sparcml_tensors_prepare.argtypes = [i32, ctypes.POINTER(Tensor), i32, i32, i32, ctypes.POINTER(Tensors), vp,
                                          ctypes.c_size_t, vp]
    L.sparcml_tensors_prepare.restype = i32
    L.sparcml_grad_norm.argtypes = [ctypes.POINTER(Tensors), ctypes.c_double, ctypes.c_double, vp, vp]
    L.sparcml_grad_norm.restype = i32
    L.sparcml_adamw.argtypes = [ctypes.POINTER(Tensors), ctypes.POINTER(AdamwArgs), vp, vp]
    L.sparcml_adamw.restype = i32
    L.sparcml_token_logprob.argtypes = [ctypes.POINTER(Logits), vp, vp, vp, ctypes.c_size_t, vp]
    L.sparcml_token_logprob.restype = i32
    L.sparcml_policy_loss.argtypes = [ctypes.POINTER(Logits), ctypes.POINTER(PolicyArgs), vp, vp, vp, u64, vp,
                                      ctypes.c_size_t, vp]
    L.sparcml_policy_loss.restype = i32
    L.sparcml_preference_loss.argtypes = [ctypes.POINTER(Logits), i32, ctypes.POINTER(u64), vp, f32, f32, f32, vp, vp,
                                          vp, u64, vp, ctypes.c_size_t, vp]
    L.sparcml_preference_loss.restype = i32
    L.sparcml_timing_enable.argtypes = [i32]
    L.sparcml_timing_enable.restype = i32
    L.sparcml_timing_read.argtypes = [i32, ctypes.POINTER(ctypes.c_float)]
    L.sparcml_timing_read.restype = i32
    L.sparcml_strerror.argtypes = [i32]
    L.sparcml_strerror.restype = ctypes.c_char_p
    L.sparcml_last_error.argtypes = []
    L.sparcml_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


TIMER_REDUCE_PASS, TIMER_REDUCE_WRITE, TIMER_REDUCE_SLOW = 0, 1, 2
TIMER_QUANT_NORM, TIMER_QUANT_CODES, TIMER_TOPK_SELECT, TIMER_TOPK_WRITE, TIMER_DENSIFY = 3, 4, 5, 6, 7
TIMER_CONCAT, TIMER_TOPK_BUCKETED, TIMER_REDUCE_MERGE = 8, 9, 10
TIMER_GRAD_NORM, TIMER_ADAMW, TIMER_LOSS_ROWS, TIMER_LOSS_GRAD = 11, 12, 13, 14


def timing_enable(on: bool) -> None:
    lib().sparcml_timing_enable(1 if on else 0)


def timing_read(group: int):
    """Mean duration (ms) of a kernel group's launches since timing was
    enabled, or None."""
    ms = ctypes.c_float(0.0)
    rc = lib().sparcml_timing_read(group, ctypes.byref(ms))
    return float(ms.value) if rc == OK else None


def strerror(status: int) -> str:
    return lib().sparcml_strerror(status).decode()


def last_error() -> str:
    return lib().sparcml_last_error().decode()


def _check(rc: int, where: str) -> None:
    if rc != OK:
        raise SparcmlError(rc, where)


def workspace_size(op: int, P: int, N: int, max_nnz: int, delta: float = 1.0) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().sparcml_workspace_size(op, P, N, max_nnz, float(delta), ctypes.byref(n)),
           "sparcml_workspace_size")
    return int(n.value)


# ---------------------------------------------------------------------------
# torch-facing helpers (device memory and streams only)

def _torch():
    import torch
    return torch


def _stream_ptr(device) -> int:
    """The current stream of a device as a hipStream_t.  (torch's own accessor
    of the raw handle: building a Stream object takes 2 us of a small call.)"""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None or device.index is None:
        return int(torch.cuda.current_stream(device).cuda_stream)
    return int(raw(device.index))


def _ptr(t) -> int:
    return int(t.data_ptr()) if t is not None and t.numel() else 0


def _require_cuda(t, name: str):
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def alloc_workspace(nbytes: int, device):
    torch = _torch()
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def topk_sparsify(x, k: int, residual=None, ws=None):
    """Per-row top-k by magnitude of x[P, N] (fp32).  residual: None, "inplace"
    (x itself becomes the residual) or a [P, N] fp32 tensor.
    Returns (idx int32 [P, k], val fp32 [P, k])."""
    torch = _torch()
    _require_cuda(x, "x")
    if x.dtype != torch.float32 or x.dim() != 2:
        raise ValueError("x must be a 2-D float32 tensor")
    P, N = x.shape
    idx = torch.empty((P, max(k, 1)), dtype=torch.int32, device=x.device)
    val = torch.empty((P, max(k, 1)), dtype=torch.float32, device=x.device)
    res_ptr = 0
    if isinstance(residual, str):
        if residual != "inplace":
            raise ValueError("residual must be None, 'inplace' or a tensor")
        res_ptr = _ptr(x)
    elif residual is not None:
        _require_cuda(residual, "residual")
        res_ptr = _ptr(residual)
    nbytes = workspace_size(OP_TOPK, P, N, k)
    if ws is None or ws.numel() < nbytes:
        ws = alloc_workspace(nbytes, x.device)
    _check(lib().sparcml_topk_sparsify(P, _ptr(x), N, k, _ptr(idx), _ptr(val), res_ptr,
                                        _ptr(ws), ws.numel(), _stream_ptr(x.device)),
           "sparcml_topk_sparsify")
    return idx[:, :k], val[:, :k]


class TopkBucketedCall:
    """Repeated bucketed top-k with error feedback (§8.4, Alg. 1) of fixed
    device rows: eps [P, N] is updated in place; idx / val [P, K]."""

    def __init__(self, eps, grad, alpha: float, bucket: int, kb: int):
        torch = _torch()
        _require_cuda(eps, "eps")
        if eps.dim() != 2 or not eps.is_contiguous() or eps.dtype != torch.float32:
            raise ValueError("eps must be a contiguous fp32 [P, N] tensor")
        if grad is not None and (grad.shape != eps.shape or not grad.is_contiguous()
                                 or grad.dtype != torch.float32):
            raise ValueError("grad must be a contiguous fp32 tensor shaped like eps")
        self.P, self.N = eps.shape
        self.eps, self.grad = eps, grad
        self.alpha, self.bucket, self.kb = float(alpha), bucket, kb
        self.K = int(lib().sparcml_topk_bucketed_count(self.N, bucket, kb))
        self.idx = torch.empty((self.P, max(self.K, 1)), dtype=torch.int32, device=eps.device)
        self.val = torch.empty((self.P, max(self.K, 1)), dtype=torch.float32, device=eps.device)

    def run(self) -> None:
        _check(lib().sparcml_topk_bucketed(self.P, _ptr(self.grad), _ptr(self.eps), self.N, self.alpha,
                                           self.bucket, self.kb, _ptr(self.idx), _ptr(self.val),
                                           _stream_ptr(self.eps.device)), "sparcml_topk_bucketed")


def topk_bucketed(eps, grad, alpha: float, bucket: int, kb: int):
    """acc = eps + alpha * grad; the kb largest magnitudes of every bucket of
    ``bucket`` coordinates; eps <- acc with them zeroed (in place).  Returns
    (idx [P, K] int32, val [P, K] fp32)."""
    c = TopkBucketedCall(eps, grad, alpha, bucket, kb)
    c.run()
    return c.idx[:, : c.K], c.val[:, : c.K]


def quantize(vals, bits: int, seed: int, want_deq: bool = False, ws=None):
    """QSGD of each fp32 tensor in ``vals``.  Returns (codes list of uint8
    tensors, scales fp32 [P], dequantized list or None)."""
    return _quantize(vals, bits, seed, want_deq, ws, 0)


def quantize_bucketed(vals, bits: int, bucket: int, seed: int, want_deq: bool = False, ws=None):
    """QSGD in buckets of ``bucket`` entries (§6).  Returns (codes list,
    flat scales fp32 -- stream r's ceil(n_r / bucket) after those of streams
    0..r-1 --, dequantized list or None)."""
    return _quantize(vals, bits, seed, want_deq, ws, bucket)


def _quantize(vals, bits, seed, want_deq, ws, bucket):
    torch = _torch()
    P = len(vals)
    dev = vals[0].device
    per = 8 // bits
    arr = (Stream * P)()
    codes, deqs = [], []
    for r, v in enumerate(vals):
        _require_cuda(v, f"vals[{r}]")
        n = v.numel()
        arr[r] = Stream(None, _ptr(v), None, None, n, 0, 0)
        codes.append(torch.empty(max((n + per - 1) // per, 1), dtype=torch.uint8, device=dev))
        if want_deq:
            deqs.append(torch.empty(max(n, 1), dtype=torch.float32, device=dev))
    qptr = (ctypes.c_void_p * P)(*[_ptr(c) for c in codes])
    dptr = (ctypes.c_void_p * P)(*[_ptr(d) for d in deqs]) if want_deq else None
    dp = ctypes.cast(dptr, ctypes.c_void_p) if dptr else None
    if bucket:
        nscale = sum((v.numel() + bucket - 1) // bucket for v in vals)
        scale = torch.empty(max(nscale, 1), dtype=torch.float32, device=dev)
        nbytes = workspace_size(OP_QUANTIZE_BUCKETED, P, 1, 0)
    else:
        nscale = P
        scale = torch.empty(P, dtype=torch.float32, device=dev)
        nbytes = workspace_size(OP_QUANTIZE, P, 1, max(v.numel() for v in vals))
    if ws is None or ws.numel() < nbytes:
        ws = alloc_workspace(nbytes, dev)
    if bucket:
        _check(lib().sparcml_quantize_bucketed(P, arr, bits, bucket, seed & (2**64 - 1),
                                               ctypes.cast(qptr, ctypes.c_void_p), _ptr(scale), dp,
                                               _ptr(ws), ws.numel(), _stream_ptr(dev)),
               "sparcml_quantize_bucketed")
    else:
        _check(lib().sparcml_quantize(P, arr, bits, seed & (2**64 - 1), ctypes.cast(qptr, ctypes.c_void_p),
                                      _ptr(scale), dp, _ptr(ws), ws.numel(), _stream_ptr(dev)),
               "sparcml_quantize")
    nb = [(v.numel() + per - 1) // per for v in vals]
    return ([c[:m] for c, m in zip(codes, nb)], scale[:nscale],
            [d[: v.numel()] for d, v in zip(deqs, vals)] if want_deq else None)


def make_streams(idx, vals=None, codes=None, scales=None, qbits: int = 0):
    """Descriptor array for P sparse streams (fp32 values or QSGD codes)."""
    P = len(idx)
    arr = (Stream * P)()
    for r in range(P):
        _require_cuda(idx[r], f"idx[{r}]")
        n = idx[r].numel()
        if qbits:
            arr[r] = Stream(_ptr(idx[r]), None, _ptr(codes[r]), int(scales[r].data_ptr()), n, 0, qbits)
        else:
            arr[r] = Stream(_ptr(idx[r]), _ptr(vals[r]), None, None, n, 0, 0)
    return arr


def sparse_reduce(idx, vals, N: int, delta: float, codes=None, scales=None, qbits: int = 0,
                  node_info: bool = False, ws=None, out_idx=None, out_val=None):
    """Sum of P sparse streams in recursive-doubling order with the dense
    switch.  ``scales`` is a device fp32 tensor [P] (one scale per stream)
    when ``qbits`` != 0.  Returns dict(idx, val, nnz, dense, node_nnz,
    node_dense); ``idx`` is None for a dense root."""
    return _reduce(idx, vals, N, None, delta, codes, scales, qbits, node_info, ws, out_idx, out_val)


def sparse_reduce_range(idx, vals, N: int, lo: int, hi: int, delta: float, codes=None, scales=None,
                        qbits: int = 0, node_info: bool = False, ws=None, out_idx=None, out_val=None):
    """One share of the split phase: the sum of P streams whose indices lie
    in [lo, hi), reduced as a vector of hi - lo (threshold floor(delta *
    (hi - lo))).  A dense root's ``val`` holds hi - lo values (index lo + i
    at i); a sparse root's ``idx`` holds absolute indices."""
    return _reduce(idx, vals, N, (lo, hi), delta, codes, scales, qbits, node_info, ws, out_idx, out_val)


def _reduce(idx, vals, N, rng, delta, codes, scales, qbits, node_info, ws, out_idx, out_val):
    torch = _torch()
    P = len(idx)
    dev = idx[0].device
    if qbits:
        scale_views = [scales[r: r + 1] for r in range(P)]
        arr = make_streams(idx, codes=codes, scales=scale_views, qbits=qbits)
    else:
        arr = make_streams(idx, vals)
    nnz = [t.numel() for t in idx]
    R = N if rng is None else rng[1] - rng[0]
    thr = int(float(delta) * float(R) // 1)
    cap = max(1, min(thr, sum(nnz)) if P > 1 else max(nnz[0], 1))
    if out_idx is None:
        out_idx = torch.empty(cap, dtype=torch.int32, device=dev)
    if out_val is None:
        out_val = torch.empty(R, dtype=torch.float32, device=dev)
    out = Stream(_ptr(out_idx), _ptr(out_val), None, None, out_idx.numel(), 0, 0)
    node_nnz = node_dense = None
    if node_info and P > 1:
        node_nnz = torch.empty(P - 1, dtype=torch.int64, device=dev)
        node_dense = torch.empty(P - 1, dtype=torch.uint8, device=dev)
    nbytes = workspace_size(OP_REDUCE, P, R, min(max(nnz), R), delta)
    if ws is None or ws.numel() < nbytes:
        ws = alloc_workspace(nbytes, dev)
    if rng is None:
        rc = lib().sparcml_sparse_reduce(P, arr, N, float(delta), ctypes.byref(out), _ptr(node_nnz),
                                         _ptr(node_dense), _ptr(ws), ws.numel(), _stream_ptr(dev))
        _check(rc, "sparcml_sparse_reduce")
    else:
        rc = lib().sparcml_sparse_reduce_range(P, arr, N, rng[0], rng[1], float(delta), ctypes.byref(out),
                                               _ptr(node_nnz), _ptr(node_dense), _ptr(ws), ws.numel(),
                                               _stream_ptr(dev))
        _check(rc, "sparcml_sparse_reduce_range")
    n = int(out.nnz)
    dense = bool(out.is_dense)
    return {
        "idx": None if dense else out_idx[:n],
        "val": out_val if dense else out_val[:n],
        "nnz": n,
        "dense": dense,
        "node_nnz": node_nnz,
        "node_dense": node_dense,
    }


class ConcatCall:
    """Repeated concatenation of P parts with disjoint index ranges (the
    gathered shares of the split-allgather allreduce) into fixed outputs.
    ``parts``: dicts with ``idx`` (device int32 tensor, or None for a dense
    part) and ``val`` (fp32) or ``codes`` + ``scales`` (QSGD, ``qbits``)."""

    def __init__(self, parts, bounds, N: int, delta: float, qbits: int = 0, bucket: int = 0):
        torch = _torch()
        self.P = len(parts)
        self.N, self.delta, self.bucket = N, float(delta), bucket
        self.dev = None
        self.arr = (Stream * self.P)()
        total = 0
        for p, part in enumerate(parts):
            n = bounds[p + 1] - bounds[p] if part["idx"] is None else part["idx"].numel()
            ref = part["codes"] if qbits else part["val"]
            _require_cuda(ref, f"parts[{p}]")
            self.dev = ref.device
            self.arr[p] = Stream(None if part["idx"] is None else _ptr(part["idx"]),
                                 None if qbits else _ptr(part["val"]),
                                 _ptr(part["codes"]) if qbits else None,
                                 _ptr(part["scales"]) if qbits else None,
                                 n, 1 if part["idx"] is None else 0, qbits)
            total += 0 if part["idx"] is None else n
        self.bounds = (ctypes.c_uint64 * (self.P + 1))(*[int(b) for b in bounds])
        self.out_idx = torch.empty(max(total, 1), dtype=torch.int32, device=self.dev)
        self.out_val = torch.empty(N, dtype=torch.float32, device=self.dev)
        self.ws = alloc_workspace(workspace_size(OP_CONCAT, self.P, N, 0), self.dev)
        self.out = Stream(_ptr(self.out_idx), _ptr(self.out_val), None, None, self.out_idx.numel(), 0, 0)
        self._keep = parts

    def run(self):
        """Returns (nnz, dense)."""
        self.out.nnz = self.out_idx.numel()
        _check(lib().sparcml_concat(self.P, self.arr, self.bounds, self.N, self.delta, self.bucket,
                                    ctypes.byref(self.out), _ptr(self.ws), self.ws.numel(),
                                    _stream_ptr(self.dev)), "sparcml_concat")
        return int(self.out.nnz), bool(self.out.is_dense)


def concat(parts, bounds, N: int, delta: float, qbits: int = 0, bucket: int = 0):
    """Concatenation of parts with disjoint index ranges (see ConcatCall).
    Returns dict(idx, val, nnz, dense); ``idx`` is None for a dense result."""
    c = ConcatCall(parts, bounds, N, delta, qbits, bucket)
    n, dense = c.run()
    return {"idx": None if dense else c.out_idx[:n], "val": c.out_val if dense else c.out_val[:n],
            "nnz": n, "dense": dense}


def validate_streams(idx, lo: int, hi: int):
    """Check that every index tensor (device int32 holding uint32 indices)
    ascends strictly inside [lo, hi).  Returns (True, "") or (False, the
    library's message naming the first offending stream and position)."""
    P = len(idx)
    arr = (Stream * P)()
    for r, t in enumerate(idx):
        _require_cuda(t, f"idx[{r}]")
        arr[r] = Stream(_ptr(t), None, None, None, t.numel(), 0, 0)
    ws = alloc_workspace(workspace_size(OP_VALIDATE, P, 1, 0), idx[0].device)
    rc = lib().sparcml_validate_streams(P, arr, lo, hi, _ptr(ws), ws.numel(), _stream_ptr(idx[0].device))
    if rc == EUNSORTED:
        return False, last_error()
    _check(rc, "sparcml_validate_streams")
    return True, ""


def split_bounds(P: int, N: int):
    """Bounds of the P index ranges of the split phase (App. A's rule:
    floor(N/P) indices per node, the rest to the last).  List of P + 1."""
    b = (ctypes.c_uint64 * (P + 1))()
    _check(lib().sparcml_split_bounds(P, N, b), "sparcml_split_bounds")
    return [int(v) for v in b]


def densify(idx, val, N: int, codes=None, scale=None, qbits: int = 0):
    """Dense fp32[N] of one sparse stream (values or QSGD codes)."""
    torch = _torch()
    dev = idx.device
    if qbits:
        s = Stream(_ptr(idx), None, _ptr(codes), int(scale.data_ptr()), idx.numel(), 0, qbits)
    else:
        s = Stream(_ptr(idx), _ptr(val), None, None, idx.numel(), 0, 0)
    out = torch.empty(N, dtype=torch.float32, device=dev)
    _check(lib().sparcml_densify(ctypes.byref(s), N, _ptr(out), _stream_ptr(dev)), "sparcml_densify")
    return out


# ---------------------------------------------------------------------------
# Prepared calls: descriptors and buffers built once, each run() is a single
# C-ABI call (used by the benchmark so that Python marshalling stays out of
# the timed loop).

class QuantizeCall:
    """Repeated QSGD of fixed device arrays into fixed code buffers
    (``bucket`` > 0: buckets of that many entries, flat scales)."""

    def __init__(self, vals, codes, scale, bits: int, seed: int, deq=None, bucket: int = 0):
        self.P = len(vals)
        self.bits, self.seed, self.bucket = bits, seed & (2**64 - 1), bucket
        self.dev = vals[0].device
        self.arr = (Stream * self.P)()
        for r, v in enumerate(vals):
            _require_cuda(v, f"vals[{r}]")
            self.arr[r] = Stream(None, _ptr(v), None, None, v.numel(), 0, 0)
        self.qptr = (ctypes.c_void_p * self.P)(*[_ptr(c) for c in codes])
        self.dptr = (ctypes.c_void_p * self.P)(*[_ptr(d) for d in deq]) if deq else None
        self.scale = scale
        if bucket:
            nbytes = workspace_size(OP_QUANTIZE_BUCKETED, self.P, 1, 0)
        else:
            nbytes = workspace_size(OP_QUANTIZE, self.P, 1, max(v.numel() for v in vals))
        self.ws = alloc_workspace(nbytes, self.dev)
        self._keep = (vals, codes, deq)

    def run(self) -> None:
        dp = ctypes.cast(self.dptr, ctypes.c_void_p) if self.dptr else None
        qp = ctypes.cast(self.qptr, ctypes.c_void_p)
        if self.bucket:
            _check(lib().sparcml_quantize_bucketed(
                self.P, self.arr, self.bits, self.bucket, self.seed, qp, _ptr(self.scale), dp,
                _ptr(self.ws), self.ws.numel(), _stream_ptr(self.dev)), "sparcml_quantize_bucketed")
        else:
            _check(lib().sparcml_quantize(
                self.P, self.arr, self.bits, self.seed, qp, _ptr(self.scale), dp,
                _ptr(self.ws), self.ws.numel(), _stream_ptr(self.dev)), "sparcml_quantize")


class ReduceCall:
    """Repeated sparse reduce of fixed device streams into fixed outputs."""

    def __init__(self, idx, N: int, delta: float, vals=None, codes=None, scales=None,
                 qbits: int = 0, node_info: bool = False, lo: int | None = None, hi: int | None = None):
        """``lo``, ``hi``: reduce the index range [lo, hi) (the split-phase
        share) instead of the whole vector."""
        self.P = len(idx)
        self.N, self.delta = N, float(delta)
        self.rng = None if lo is None else (int(lo), int(hi))
        R = N if self.rng is None else self.rng[1] - self.rng[0]
        self.dev = idx[0].device
        torch = _torch()
        if qbits:
            self.arr = make_streams(idx, codes=codes, scales=[scales[r: r + 1] for r in range(self.P)],
                                    qbits=qbits)
        else:
            self.arr = make_streams(idx, vals)
        nnz = [t.numel() for t in idx]
        thr = int(self.delta * float(R) // 1)
        cap = max(1, min(thr, sum(nnz)) if self.P > 1 else max(nnz[0], 1))
        self.out_idx = torch.empty(cap, dtype=torch.int32, device=self.dev)
        self.out_val = torch.empty(R, dtype=torch.float32, device=self.dev)
        self.node_nnz = self.node_dense = None
        if node_info and self.P > 1:
            self.node_nnz = torch.empty(self.P - 1, dtype=torch.int64, device=self.dev)
            self.node_dense = torch.empty(self.P - 1, dtype=torch.uint8, device=self.dev)
        nbytes = workspace_size(OP_REDUCE, self.P, R, min(max(nnz), R), self.delta)
        self.ws = alloc_workspace(nbytes, self.dev)
        self.out = Stream(_ptr(self.out_idx), _ptr(self.out_val), None, None, self.out_idx.numel(), 0, 0)
        self._keep = (idx, vals, codes, scales)

    def run_async(self):
        """Enqueue the reduction without waiting (capturable in a HIP
        graph); the root header lands in ``self.result`` (device int64 [2]:
        nnz, dense flag in the low word of the second)."""
        if not hasattr(self, "result"):
            torch = _torch()
            self.result = torch.zeros(2, dtype=torch.int64, device=self.dev)
        self.out.nnz = self.out_idx.numel()
        lo, hi = self.rng if self.rng is not None else (0, self.N)
        _check(lib().sparcml_sparse_reduce_async(
            self.P, self.arr, self.N, lo, hi, self.delta, ctypes.byref(self.out), _ptr(self.node_nnz),
            _ptr(self.node_dense), _ptr(self.result), _ptr(self.ws), self.ws.numel(),
            _stream_ptr(self.dev)), "sparcml_sparse_reduce_async")

    def run_async_noalloc(self):
        """run_async through the allocation-free entry point (the library's
        fixed scratch array instead of ``self.ws``)."""
        if not hasattr(self, "result"):
            torch = _torch()
            self.result = torch.zeros(2, dtype=torch.int64, device=self.dev)
        self.out.nnz = self.out_idx.numel()
        lo, hi = self.rng if self.rng is not None else (0, self.N)
        _check(lib().sparcml_sparse_reduce_async_noalloc(
            self.P, self.arr, self.N, lo, hi, self.delta, ctypes.byref(self.out), _ptr(self.node_nnz),
            _ptr(self.node_dense), _ptr(self.result), _stream_ptr(self.dev)),
            "sparcml_sparse_reduce_async_noalloc")

    def result_header(self):
        """(nnz, dense) from ``self.result`` (synchronizes); raises if the
        header's reserved word reports an incomplete reduction."""
        r = self.result.cpu()
        flags = (int(r[1]) >> 32) & 0xFFFFFFFF
        if flags & 2:
            raise RuntimeError("sparse_reduce_async: the merge path met streams that do not ascend; "
                               "the outputs are incomplete")
        if flags:
            raise RuntimeError("sparse_reduce_async: a segment of the merge path gave up waiting for its "
                               "predecessors' sizes; the outputs are incomplete")
        return int(r[0]), bool(int(r[1]) & 0xFFFFFFFF)

    def run(self):
        """Returns (nnz, dense)."""
        self.out.nnz = self.out_idx.numel()
        if self.rng is None:
            _check(lib().sparcml_sparse_reduce(
                self.P, self.arr, self.N, self.delta, ctypes.byref(self.out), _ptr(self.node_nnz),
                _ptr(self.node_dense), _ptr(self.ws), self.ws.numel(), _stream_ptr(self.dev)),
                "sparcml_sparse_reduce")
        else:
            _check(lib().sparcml_sparse_reduce_range(
                self.P, self.arr, self.N, self.rng[0], self.rng[1], self.delta, ctypes.byref(self.out),
                _ptr(self.node_nnz), _ptr(self.node_dense), _ptr(self.ws), self.ws.numel(),
                _stream_ptr(self.dev)), "sparcml_sparse_reduce_range")
        return int(self.out.nnz), bool(self.out.is_dense)


class TopkCall:
    """Repeated top-k of a fixed device matrix into fixed outputs."""

    def __init__(self, x, k: int, residual=None):
        torch = _torch()
        _require_cuda(x, "x")
        self.x, self.k = x, k
        self.P, self.N = x.shape
        self.idx = torch.empty((self.P, max(k, 1)), dtype=torch.int32, device=x.device)
        self.val = torch.empty((self.P, max(k, 1)), dtype=torch.float32, device=x.device)
        self.res_ptr = _ptr(residual) if residual is not None else 0
        nbytes = workspace_size(OP_TOPK, self.P, self.N, k)
        self.ws = alloc_workspace(nbytes, x.device)
        self._keep = residual

    def run(self) -> None:
        _check(lib().sparcml_topk_sparsify(
            self.P, _ptr(self.x), self.N, self.k, _ptr(self.idx), _ptr(self.val), self.res_ptr,
            _ptr(self.ws), self.ws.numel(), _stream_ptr(self.x.device)), "sparcml_topk_sparsify")


# ---------------------------------------------------------------------------
# Training operators: the losses that a gradient comes from, the update that
# the summed gradient goes into.

STATE_BLOCK = 256  # elements that share a scale (8-bit moments)


def _type_id(t, name: str) -> int:
    torch = _torch()
    ids = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
    if t.dtype not in ids:
        raise ValueError(f"{name} must be float32, bfloat16 or float16")
    return ids[t.dtype]


def _require(t, name: str, dtype, numel: int, device) -> None:
    _require_cuda(t, name)
    if t.dtype != dtype or t.numel() != numel or t.device != device:
        raise ValueError(f"{name} must hold {numel} {dtype} entries on {device}")


def adamw_state(params, state_bits: int = 32):
    """Moments of a model at the start of training: (m, v) lists of fp32
    tensors, or (m, v, m_scale, v_scale) with E4M3 codes and a scale per 256
    elements (``state_bits`` 8), all zero."""
    torch = _torch()
    if state_bits == 32:
        return [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params]
    if state_bits != 8:
        raise ValueError("state_bits must be 8 or 32")
    codes = lambda: [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)  # noqa: E731
                     for p in params]
    scales = lambda: [torch.zeros(-(-p.numel() // STATE_BLOCK), device=p.device) for p in params]  # noqa: E731
    return codes(), codes(), scales(), scales()


def _pointers(tensors, name: str, dtypes, numels, index: int, what: str):
    """Addresses of one list of a model's tensors, each checked."""
    # whole lists at once: a large model has a thousand tensors
    torch = _torch()
    fine = (all(isinstance(x, torch.Tensor) for x in tensors) and {x.dtype for x in tensors} <= set(dtypes)
            and {x.get_device() for x in tensors} == {index} and all([x.is_contiguous() for x in tensors]))
    if not fine or [x.numel() for x in tensors] != numels:
        t = next((t for t, (x, n) in enumerate(zip(tensors, numels)) if not isinstance(x, torch.Tensor)
                  or x.dtype not in dtypes or x.get_device() != index or not x.is_contiguous() or x.numel() != n), 0)
        raise ValueError(f"{name}[{t}] must be a contiguous tensor of {numels[t]} {what} on the gradients' device")
    return [x.data_ptr() for x in tensors]


class _TensorPlan:
    """A prepared plan of a model's tensors and its workspace.  ``columns``
    (from the sizes and the device's index): the descriptors' other fields."""

    def __init__(self, grads, state_bits=0, copy_type=BF16, columns=None):
        torch = _torch()
        if not grads:
            raise ValueError("no tensors")
        _require_cuda(grads[0], "grads[0]")
        self.dev = grads[0].device
        gtype = _type_id(grads[0], "grads[0]")
        sizes = [g.numel() for g in grads]
        fields = {"grad": _pointers(grads, "grads", (grads[0].dtype,), sizes, grads[0].get_device(),
                                    f"{grads[0].dtype} gradients"), "n": sizes}
        if columns:
            fields.update(columns(sizes, grads[0].get_device()))
        # packed from columns: setting fields one by one takes a microsecond a tensor
        none = [0] * len(grads)
        rates = (array.array("f", fields.pop(name, none)) for name in _TENSOR_COLUMNS[8:])
        arr = ctypes.c_char_p(b"".join(map(_pack_tensor, *(fields.get(name, none) for name in _TENSOR_COLUMNS[:8]), *rates)))
        self.plan = Tensors()
        self.ws = alloc_workspace(workspace_size(OP_TENSORS, len(grads), sum(sizes), 0), self.dev)
        _check(lib().sparcml_tensors_prepare(len(grads), ctypes.cast(arr, ctypes.POINTER(Tensor)), gtype, copy_type,
                                             state_bits, ctypes.byref(self.plan), _ptr(self.ws), self.ws.numel(),
                                             _stream_ptr(self.dev)), "sparcml_tensors_prepare")
        self.out = torch.empty(2, dtype=torch.float32, device=self.dev)
        self._plan, self._out = ctypes.byref(self.plan), self.out.data_ptr()

    def _norm(self, max_norm, grad_scale):
        _check(lib().sparcml_grad_norm(self._plan, grad_scale, max_norm, self._out, _stream_ptr(self.dev)),
               "sparcml_grad_norm")


class GradNormCall(_TensorPlan):
    """Repeated norm of a list of gradients (fp32, bf16 or fp16, one type):
    run() fills ``out`` (device fp32 [2]) with the norm and the factor
    min(1, max_norm / norm) that clips it (0 if the norm is not finite)."""

    def __init__(self, grads):
        super().__init__(grads)
        self._keep = grads

    def run(self, max_norm: float = float("inf"), grad_scale: float = 1.0) -> None:
        self._norm(max_norm, grad_scale)


def grad_norm(grads, max_norm: float = float("inf"), grad_scale: float = 1.0):
    """Norm of all gradients and the factor that clips it (device fp32 [2])."""
    c = GradNormCall(grads)
    c.run(max_norm, grad_scale)
    return c.out


class AdamwCall(_TensorPlan):
    """AdamW over a fixed set of tensors.  ``params``, ``grads``, ``m``, ``v``:
    lists of contiguous tensors (fp32 weights; fp32, bf16 or fp16 gradients;
    moments fp32, or one-byte codes with ``m_scale`` / ``v_scale``, as
    adamw_state makes them).  ``copies``: tensors of one 16-bit type that
    receive the new weights, or None (for all, or for a tensor).  ``decay``,
    ``lr_scale``: a number, or one for each tensor."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None, decay=0.0, lr_scale=1.0):
        torch = _torch()
        count = len(grads)
        bits = 8 if m_scale is not None else 32
        lists = {"params": params, "m": m, "v": v, "copies": copies, "m_scale": m_scale, "v_scale": v_scale}
        if (m_scale is None) != (v_scale is None):
            raise ValueError("m_scale and v_scale go together")
        for name, x in lists.items():
            if x is not None and len(x) != count:
                raise ValueError(f"{name} must hold {count} tensors")
        per = lambda x: [float(x)] * count if isinstance(x, (int, float)) else [float(y) for y in x]  # noqa: E731
        decay, lr_scale = per(decay), per(lr_scale)
        if len(decay) != count or len(lr_scale) != count:
            raise ValueError(f"decay and lr_scale must hold {count} numbers")
        given = [c for c in copies or [] if c is not None]
        ctype = _type_id(given[0], "copies") if given else BF16
        if ctype == F32:
            raise ValueError("copies must be bfloat16 or float16")

        def columns(sizes, index):
            moment = ((torch.float32,), "fp32 moments") if bits == 32 else (
                (torch.uint8, torch.float8_e4m3fn), "E4M3 codes")
            f = {"param": _pointers(params, "params", (torch.float32,), sizes, index, "fp32 weights"),
                 "m": _pointers(m, "m", moment[0], sizes, index, moment[1]),
                 "v": _pointers(v, "v", moment[0], sizes, index, moment[1]),
                 "decay": decay, "lr_scale": lr_scale}
            if bits == 8:
                blocks = [-(-n // STATE_BLOCK) for n in sizes]
                f["m_scale"] = _pointers(m_scale, "m_scale", (torch.float32,), blocks, index, "scales")
                f["v_scale"] = _pointers(v_scale, "v_scale", (torch.float32,), blocks, index, "scales")
            if given:
                at = iter(_pointers(given, "copies", (given[0].dtype,),
                                    [n for n, c in zip(sizes, copies) if c is not None], index, f"{given[0].dtype} entries"))
                f["copy"] = [0 if c is None else next(at) for c in copies]
            return f

        super().__init__(grads, bits, ctype, columns)
        self.args = AdamwArgs()
        self._args = ctypes.byref(self.args)
        self._keep = (params, grads, m, v, m_scale, v_scale, copies)

    def grad_norm(self, max_norm: float = float("inf"), grad_scale: float = 1.0):
        """Norm of the gradients and the factor that clips it, in ``out``
        (device fp32 [2]), for run's ``clip``."""
        self._norm(max_norm, grad_scale)
        return self.out

    def run(self, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
            grad_scale: float = 1.0, clip=None, seed: int = 0) -> None:
        """Step number ``step`` (from 1 on), in place.  ``clip``: a device
        tensor as grad_norm fills it, or None."""
        if clip is not None:
            _require(clip, "clip", _torch().float32, 2, self.dev)
        if not 1 <= step < 2**32:
            raise ValueError("step must be in [1, 2^32)")
        a = self.args
        a.lr, a.beta1, a.beta2, a.eps, a.grad_scale = lr, beta1, beta2, eps, grad_scale
        a.seed, a.step = seed & (2**64 - 1), step
        _check(lib().sparcml_adamw(self._plan, self._args, None if clip is None else clip.data_ptr(),
                                   _stream_ptr(self.dev)), "sparcml_adamw")


class _LogitsCall:
    def __init__(self, logits, labels, scale, op, pairs=1):
        torch = _torch()
        if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
            raise ValueError("logits must be a CUDA (HIP) tensor")
        if logits.dim() != 2 or not logits.numel() or (logits.stride(1) != 1 and logits.shape[1] > 1):
            raise ValueError("logits must be a 2-D tensor with adjacent columns")
        self.rows, self.vocab = logits.shape
        self.dev = logits.device
        ld = logits.stride(0) if self.rows > 1 else self.vocab
        _require(labels, "labels", torch.int32, self.rows, self.dev)
        self.logits = Logits(logits.data_ptr(), _ptr(labels), self.rows, self.vocab, ld, _type_id(logits, "logits"),
                             scale)
        self.ws = alloc_workspace(workspace_size(op, pairs, self.rows, self.vocab), self.dev)
        self.logp = torch.empty(self.rows, dtype=torch.float32, device=self.dev)
        self._keep = [logits, labels]
        # what every run passes
        self._in, self._logp = ctypes.byref(self.logits), self.logp.data_ptr()
        self._ws = (self.ws.data_ptr(), self.ws.numel())

    def _per_row(self, t, name):
        if t is not None:
            _require(t, name, _torch().float32, self.rows, self.dev)
            self._keep.append(t)
        return _ptr(t)

    def _gradient(self, dlogits):
        """Place of the gradient: a new tensor, "inplace", None or a tensor."""
        torch = _torch()
        logits = self._keep[0]
        if isinstance(dlogits, str):
            if dlogits not in ("new", "inplace"):
                raise ValueError("dlogits must be 'new', 'inplace', None or a tensor")
            dlogits = logits if dlogits == "inplace" else torch.empty(self.rows, self.vocab, dtype=logits.dtype,
                                                                      device=self.dev)
        if dlogits is not None:
            if (dlogits.shape != logits.shape or dlogits.dtype != logits.dtype or dlogits.device != self.dev
                    or (dlogits.stride(1) != 1 and self.vocab > 1)):
                raise ValueError("dlogits must have the logits' shape, type and adjacent columns")
            self._ldd = dlogits.stride(0) if self.rows > 1 else self.vocab
        else:
            self._ldd = 0
        self.dlogits = dlogits
        self.stats = torch.empty(4, dtype=torch.float32, device=self.dev)
        self._outs = (self._logp, self.stats.data_ptr(), _ptr(dlogits), self._ldd, *self._ws)


class TokenLogprobCall(_LogitsCall):
    """Repeated log probability of each row's token: logits [T, V] (fp32, bf16
    or fp16, rows at any stride), labels int32 [T] (outside [0, V): no token);
    run() fills ``logp`` and ``lse`` (fp32 [T]; 0 without a token)."""

    def __init__(self, logits, labels, scale: float = 1.0):
        super().__init__(logits, labels, scale, OP_LOGPROB)
        self.lse = _torch().empty_like(self.logp)
        self._outs = (self._logp, self.lse.data_ptr(), *self._ws)

    def run(self) -> None:
        _check(lib().sparcml_token_logprob(self._in, *self._outs, _stream_ptr(self.dev)), "sparcml_token_logprob")


def token_logprob(logits, labels, scale: float = 1.0):
    """Log probability of each row's token under softmax(scale * logits) and
    the rows' log sums: (logp, lse), fp32 [T]."""
    c = TokenLogprobCall(logits, labels, scale)
    c.run()
    return c.logp, c.lse


class PolicyLossCall(_LogitsCall):
    """Repeated clipped policy loss with a KL term.  ``old``, ``adv``,
    ``weight``, ``ref`` (or None): fp32 [T]; a row of weight 0 counts for
    nothing and is not read.  run() fills ``stats`` (loss, its clipped part,
    KL, clipped share), ``logp`` and ``dlogits`` ("new", "inplace": the
    logits' own place, a tensor, or None: forward only)."""

    def __init__(self, logits, labels, old, adv, weight, ref=None, clip_lo: float = 0.2, clip_hi: float = 0.2,
                 kl: float = 0.0, scale: float = 1.0, grad_scale: float = 1.0, dlogits="new"):
        super().__init__(logits, labels, scale, OP_POLICY)
        if old is None or adv is None or weight is None:
            raise ValueError("old, adv and weight must be given")
        self.args = PolicyArgs(self._per_row(old, "old"), self._per_row(ref, "ref"), self._per_row(adv, "adv"),
                               self._per_row(weight, "weight"), clip_lo, clip_hi, kl, grad_scale)
        self._args = ctypes.byref(self.args)
        self._gradient(dlogits)

    def run(self) -> None:
        _check(lib().sparcml_policy_loss(self._in, self._args, *self._outs, _stream_ptr(self.dev)),
               "sparcml_policy_loss")


def policy_loss(logits, labels, old, adv, weight, **more):
    """One clipped policy loss and its gradient (see PolicyLossCall):
    dict(stats, logp, dlogits)."""
    c = PolicyLossCall(logits, labels, old, adv, weight, **more)
    c.run()
    return {"stats": c.stats, "logp": c.logp, "dlogits": c.dlogits}


class PreferenceLossCall(_LogitsCall):
    """Repeated loss of paired log ratios.  ``bounds``: row numbers at which
    the 2 * pairs sequences begin, and the end (of pair b, sequence 2b is the
    preferred one); ``ref``: fp32 [T] or None.  run() fills ``stats`` (loss,
    share of pairs in order, mean rewards of the preferred and the others),
    ``logp`` and ``dlogits`` (as PolicyLossCall)."""

    def __init__(self, logits, labels, bounds, ref=None, beta: float = 0.1, smoothing: float = 0.0,
                 scale: float = 1.0, grad_scale: float = 1.0, dlogits="new"):
        if len(bounds) < 3 or len(bounds) % 2 == 0:
            raise ValueError("bounds must hold 2 * pairs + 1 row numbers")
        self.pairs = len(bounds) // 2
        super().__init__(logits, labels, scale, OP_PREFERENCE, self.pairs)
        if any(int(b) < 0 for b in bounds):
            raise ValueError("bounds must not be negative")
        self.bounds = (ctypes.c_uint64 * len(bounds))(*[int(b) for b in bounds])
        self.ref = self._per_row(ref, "ref")
        self.rates = (beta, smoothing, grad_scale)
        self._gradient(dlogits)

    def run(self) -> None:
        _check(lib().sparcml_preference_loss(self._in, self.pairs, self.bounds, self.ref, *self.rates, *self._outs,
                                             _stream_ptr(self.dev)), "sparcml_preference_loss")


def preference_loss(logits, labels, bounds, **more):
    """One loss of paired log ratios and its gradient (see
    PreferenceLossCall): dict(stats, logp, dlogits)."""
    c = PreferenceLossCall(logits, labels, bounds, **more)
    c.run()
    return {"stats": c.stats, "logp": c.logp, "dlogits": c.dlogits}
