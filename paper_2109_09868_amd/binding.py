"""Binding of libapproxifer.so: same names as the C ABI, argument marshalling only.

Calls in their ordinary form (tensors and float64 node arrays as documented, outputs given, torch's current stream) are
marshalled by the compiled module _marshal; every other form, and every error, goes through ctypes below.

Tensors are torch CUDA (ROCm) tensors used purely as device buffers; every step of the
coding layer runs inside the library's HIP kernels.  There is no CPU fallback: if the
library is missing the loader raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libapproxifer.so")
MARSHAL_PATH = os.path.join(_PKG_DIR, "_marshal.so")

MAX_K = 64
MAX_N = 128
MAX_AVAIL_BYZ = 64
SIGN_WORKER_INDEX = 0
SIGN_SURVIVOR_RANK = 1
S_FROM_MASK = -1
F32, F16, BF16 = 0, 1, 2
SEQUENCE_OK, SEQUENCE_BAD, SEQUENCE_BAD_PAGE, SEQUENCE_NO_PAGES, SEQUENCE_SHARED_PAGE = range(5)

EXPORTS = (
    "approxifer_version",
    "approxifer_wait_mask",
    "approxifer_strerror",
    "approxifer_chebyshev_nodes",
    "approxifer_encode",
    "approxifer_decode",
    "approxifer_decode_top1",
    "approxifer_decode_byzantine",
    "approxifer_decode_byzantine_homogeneous",
    "approxifer_workspace_bytes",
    "approxifer_decode_byzantine_static",
    "approxifer_decode_rational",
    "approxifer_group_count",
    "approxifer_pad_last_group",
    "approxifer_top1",
    "approxifer_rotary_frequencies",
    "approxifer_append",
    "approxifer_attend",
    "approxifer_attend_workspace_bytes",
    "approxifer_cache_reserve",
    "approxifer_cache_fork",
    "approxifer_cache_compact",
    "approxifer_cache_workspace_bytes",
    "approxifer_attend_shared",
    "approxifer_attend_shared_workspace_bytes",
    "approxifer_attend_shared_pays",
    "approxifer_attend_mass",
    "approxifer_attend_mass_workspace_bytes",
    "approxifer_cache_evict",
    "approxifer_cache_evict_workspace_bytes",
)


class _Sequences(ctypes.Structure):
    """approxifer_sequences."""
    _fields_ = [("d_table", ctypes.c_void_p), ("d_lens", ctypes.c_void_p), ("d_starts", ctypes.c_void_p),
                ("T", ctypes.c_int64), ("B", ctypes.c_int64), ("M", ctypes.c_int64), ("P", ctypes.c_int64),
                ("page", ctypes.c_int32)]


_lib = None


class ApproxiferError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("approxifer error %d: %s" % (code, text))
        self.code = code


def load() -> ctypes.CDLL:
    """Load the HIP library built in-tree.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "%s is missing: build it first (python -c 'import __graft_entry__ as g; g.build()'). "
            "There is no fallback path." % LIB_PATH
        )
    lib = ctypes.CDLL(LIB_PATH)
    c_dp = ctypes.POINTER(ctypes.c_double)
    vp = ctypes.c_void_p
    lib.approxifer_version.restype = ctypes.c_int
    lib.approxifer_version.argtypes = []
    lib.approxifer_strerror.restype = ctypes.c_char_p
    lib.approxifer_strerror.argtypes = [ctypes.c_int]
    lib.approxifer_chebyshev_nodes.restype = ctypes.c_int
    lib.approxifer_chebyshev_nodes.argtypes = [ctypes.c_int, ctypes.c_int, c_dp, c_dp]
    lib.approxifer_encode.restype = ctypes.c_int
    lib.approxifer_encode.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int64, c_dp, c_dp, vp]
    lib.approxifer_decode.restype = ctypes.c_int
    lib.approxifer_decode.argtypes = [vp, vp, vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_int64, c_dp, c_dp, ctypes.c_int, vp]
    lib.approxifer_decode_top1.restype = ctypes.c_int
    lib.approxifer_decode_top1.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                           ctypes.c_int64, c_dp, c_dp, ctypes.c_int, vp]
    lib.approxifer_decode_byzantine.restype = ctypes.c_int
    lib.approxifer_decode_byzantine.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                                ctypes.c_int, ctypes.c_int, ctypes.c_int64, c_dp, c_dp, ctypes.c_int,
                                                vp, ctypes.c_size_t, vp]
    lib.approxifer_workspace_bytes.restype = ctypes.c_size_t
    lib.approxifer_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                               ctypes.c_int64]
    lib.approxifer_decode_byzantine_static.restype = ctypes.c_int
    lib.approxifer_decode_byzantine_static.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                                       ctypes.c_int, ctypes.c_int, ctypes.c_int64, c_dp, c_dp,
                                                       ctypes.c_int, vp]
    lib.approxifer_group_count.restype = ctypes.c_int64
    lib.approxifer_group_count.argtypes = [ctypes.c_int64, ctypes.c_int]
    lib.approxifer_pad_last_group.restype = ctypes.c_int
    lib.approxifer_pad_last_group.argtypes = [vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int64, vp]
    lib.approxifer_top1.restype = ctypes.c_int
    lib.approxifer_top1.argtypes = [vp, vp, vp, ctypes.c_int64, ctypes.c_int64, vp]
    lib.approxifer_decode_rational.restype = ctypes.c_int
    lib.approxifer_decode_rational.argtypes = [vp, vp, vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                               ctypes.c_int, ctypes.c_int64, c_dp, c_dp, vp]
    lib.approxifer_decode_byzantine_homogeneous.restype = ctypes.c_int
    lib.approxifer_decode_byzantine_homogeneous.argtypes = lib.approxifer_decode_byzantine.argtypes
    lib.approxifer_wait_mask.restype = ctypes.c_int
    lib.approxifer_wait_mask.argtypes = [vp, vp, vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, vp]
    i, q, f, z = ctypes.c_int, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
    seq = ctypes.POINTER(_Sequences)
    lib.approxifer_rotary_frequencies.restype = i
    lib.approxifer_rotary_frequencies.argtypes = [i, f, c_dp]
    lib.approxifer_append.restype = i
    lib.approxifer_append.argtypes = [seq, i, i, i, i, vp, q, vp, q, vp, q, vp, vp, vp, vp, vp, f, vp, i, c_dp, vp, i, i, vp, vp]
    lib.approxifer_attend.restype = i
    lib.approxifer_attend.argtypes = [seq, i, i, i, i, vp, q, vp, vp, vp, q, q, q, q, f, vp, vp, z, vp]
    lib.approxifer_attend_workspace_bytes.restype = z
    lib.approxifer_attend_workspace_bytes.argtypes = [q, q, i, i, i, i, q, q, q, q]
    lib.approxifer_cache_reserve.restype = i
    lib.approxifer_cache_reserve.argtypes = [vp, vp, vp, vp, vp, q, q, q, i, vp]
    lib.approxifer_cache_fork.restype = i
    lib.approxifer_cache_fork.argtypes = [vp] * 10 + [q] * 6 + [i, vp, z, vp]
    lib.approxifer_cache_compact.restype = i
    lib.approxifer_cache_compact.argtypes = [vp] * 6 + [q] * 5 + [i, vp, z, vp]
    lib.approxifer_cache_workspace_bytes.restype = z
    lib.approxifer_cache_workspace_bytes.argtypes = [q, q, q]
    lib.approxifer_attend_shared.restype = i
    lib.approxifer_attend_shared.argtypes = [seq, i, i, i, i, vp, q, vp, vp, vp, vp, vp, q, q, q, q, q, q, f, vp, vp, z, vp]
    lib.approxifer_attend_shared_workspace_bytes.restype = z
    lib.approxifer_attend_shared_workspace_bytes.argtypes = [q, q, q, i, i, i, i, q, q, q, q, q]
    lib.approxifer_attend_shared_pays.restype = i
    lib.approxifer_attend_shared_pays.argtypes = [q, q, q, i, i, i, i, i, q, q, q, q, q]
    lib.approxifer_attend_mass.restype = i
    lib.approxifer_attend_mass.argtypes = [seq, i, i, i, i, vp, q, vp, vp, vp, vp, q, q, q, q, q, f, vp, vp, z, vp]
    lib.approxifer_attend_mass_workspace_bytes.restype = z
    lib.approxifer_attend_mass_workspace_bytes.argtypes = lib.approxifer_attend_workspace_bytes.argtypes
    lib.approxifer_cache_evict.restype = i
    lib.approxifer_cache_evict.argtypes = [vp, vp, vp, vp, q, vp, vp, vp] + [q] * 6 + [i, q, q, q, vp, z, vp]
    lib.approxifer_cache_evict_workspace_bytes.restype = z
    lib.approxifer_cache_evict_workspace_bytes.argtypes = [q, q, q, i]
    _lib = lib
    return lib


_entries = None


def _entry() -> ctypes.CDLL:
    """The library once more, for the calls below: node arrays go in as plain addresses (here: bytes objects), so that no
    ctypes pointer object has to be built for them (3 us each, half of what a call took on the host)."""
    global _entries
    lib = load()
    if _entries is None or _entries[0] is not lib:
        fast = ctypes.CDLL(LIB_PATH)
        for name in EXPORTS:
            typed = getattr(lib, name)
            if typed.argtypes is not None:
                getattr(fast, name).argtypes = [ctypes.c_void_p if t is ctypes.POINTER(ctypes.c_double) else t
                                                for t in typed.argtypes]
            getattr(fast, name).restype = typed.restype
        _entries = (lib, fast)
    return _entries[1]


_ordinary = None      # (library, the compiled marshalling module, its handle of the library)


def marshal_target() -> str:
    """The interpreter and torch that the marshalling module is compiled for."""
    import sys

    import torch
    return "%s torch %s" % (sys.implementation.cache_tag, torch.__version__)


def _marshal_module():
    """The compiled marshalling module, or None.  One that is there but is not for this interpreter and torch, whose layouts
    are compiled into it, is not used, and a warning says so."""
    if not os.path.exists(MARSHAL_PATH):
        return None
    try:
        import torch  # noqa: F401  (the module links its libraries)
        from . import _marshal as module
        if module.built_for == marshal_target():
            return module
        why = "it was built for %s" % module.built_for
    except (ImportError, AttributeError) as e:
        why = str(e)
    import warnings
    warnings.warn("%s is not used, calls take longer on the host: %s; build it again" % (MARSHAL_PATH, why), RuntimeWarning,
                  stacklevel=2)
    return None


def _marshal():
    """The compiled marshalling module and its handle of the library, or (None, None) where it has not been built: the
    calls then go through ctypes, 3 us more each on the host (a decode of 64 groups: 6.8 us to enqueue, 3.4 with it)."""
    global _ordinary
    lib = load()
    if _ordinary is None or _ordinary[0] is not lib:
        module, handle = _marshal_module(), None
        if module is not None:
            names = ("encode", "decode", "decode_top1", "decode_byzantine", "decode_byzantine_homogeneous", "pad_last_group",
                     "top1", "wait_mask", "append", "attend", "cache_reserve", "cache_fork", "cache_compact", "cache_evict",
                     "attend_mass", "attend_shared")
            handle = module.bind(*(ctypes.cast(getattr(lib, "approxifer_" + n), ctypes.c_void_p).value for n in names))
        _ordinary = (lib, module, handle)
    return _ordinary[1], _ordinary[2]


def _done(status) -> bool:
    """Whether the compiled marshalling made the call; raises what the call returned."""
    if status is None:
        return False
    if status != 0:
        _check(status)
    return True


def strerror(code: int) -> str:
    return load().approxifer_strerror(int(code)).decode()


def _check(code: int) -> None:
    if code != 0:
        raise ApproxiferError(code, strerror(code))


def _nodes(a) -> tuple:
    """(number of nodes, their float64 values as bytes, which ctypes passes as a pointer without building one)."""
    arr = np.asarray(a, dtype=np.float64)
    return arr.size, arr.tobytes()


def _stream_handle(stream) -> int:
    if stream is None:
        import torch
        # torch.cuda.current_stream().cuda_stream without the Stream object around it; not a documented name, so the
        # documented way is there where it is missing
        try:
            return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
        except AttributeError:
            return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _dev(t, dtype, shape=None):
    """Address of a contiguous device tensor of this dtype and, where given, shape (a tuple)."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("expected a tensor in device memory")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError("expected a contiguous %s tensor, got %s" % (dtype, t.dtype))
    if shape is not None and t.shape != shape:
        raise ValueError("expected shape %s, got %s" % (tuple(shape), tuple(t.shape)))
    return t.data_ptr()


def approxifer_chebyshev_nodes(K: int, N: int):
    """(alpha[K], beta[N]) float64 numpy arrays from the library's own node generator."""
    alpha = np.empty(max(K, 0), dtype=np.float64)
    beta = np.empty(max(N, 0), dtype=np.float64)
    _check(load().approxifer_chebyshev_nodes(int(K), int(N),
                                             alpha.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                             beta.ctypes.data_as(ctypes.POINTER(ctypes.c_double))))
    return alpha, beta


def approxifer_group_count(Q: int, K: int) -> int:
    """Number of groups of K consecutive queries that a stream of Q queries forms."""
    return _entry().approxifer_group_count(int(Q), int(K))


def approxifer_pad_last_group(buffer, Q, K, stream=None):
    """buffer: [rows, D] float32 device tensor with rows >= ceil(Q / K) * K whose first Q rows hold the stream;
    rows Q .. ceil(Q / K) * K - 1 become copies of row Q - 1.  Returns the buffer's first G * K rows as [G, K, D]."""
    if stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.pad_last_group(lib, buffer, Q, K)):
            G = -(-Q // K)
            return buffer[: G * K].view(G, K, buffer.shape[1])
    import torch
    rows, D = buffer.shape
    G = approxifer_group_count(Q, K)
    if G < 0 or rows < G * K:
        raise ValueError("the buffer must hold ceil(Q / K) * K rows")
    _check(_entry().approxifer_pad_last_group(_dev(buffer, torch.float32), int(Q), int(K), int(D),
                                              _stream_handle(stream)))
    return buffer[: G * K].view(G, K, D)


def approxifer_encode(queries, alpha, beta, coded=None, stream=None):
    """queries [G, K, D] float32 device tensor -> coded [G, N, D]; K = len(alpha), N = len(beta)."""
    if coded is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.encode(lib, queries, alpha, beta, coded)):
            return coded
    import torch
    n_alpha, ap = _nodes(alpha)
    N, bp = _nodes(beta)
    G, K, D = queries.shape
    if K != n_alpha:
        raise ValueError("queries.shape[1] must equal len(alpha)")
    if coded is None:
        coded = torch.empty((G, N, D), dtype=torch.float32, device=queries.device)
    _check(_entry().approxifer_encode(_dev(queries, torch.float32), _dev(coded, torch.float32, (G, N, D)),
                                      G, K, N, D, ap, bp, _stream_handle(stream)))
    return coded


def approxifer_decode(preds, mask, alpha, beta, S, sign_mode=SIGN_WORKER_INDEX, out=None, status=None, stream=None):
    """preds [G, N, C] float32, mask [G, N] uint8 -> (out [G, K, C] float32, status [G] int32)."""
    if out is not None and status is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.decode(lib, preds, mask, alpha, beta, S, sign_mode, out, status)):
            return out, status
    import torch
    K, ap = _nodes(alpha)
    n_beta, bp = _nodes(beta)
    G, N, C = preds.shape
    if N != n_beta:
        raise ValueError("preds.shape[1] must equal len(beta)")
    if out is None:
        out = torch.zeros((G, K, C), dtype=torch.float32, device=preds.device)
    if status is None:
        status = torch.full((G,), -1, dtype=torch.int32, device=preds.device)
    _check(_entry().approxifer_decode(_dev(preds, torch.float32), _dev(mask, torch.uint8, (G, N)),
                                      _dev(out, torch.float32, (G, K, C)), _dev(status, torch.int32, (G,)),
                                      G, K, N, int(S), C, ap, bp, int(sign_mode),
                                      _stream_handle(stream)))
    return out, status


def approxifer_decode_top1(preds, mask, alpha, beta, S, sign_mode=SIGN_WORKER_INDEX, top1=None, score=None, status=None,
                           stream=None, want_score=True):
    """Fused decode + argmax over classes: (top1 [G, K] int32, score [G, K] float32 or None, status [G] int32)."""
    if top1 is not None and status is not None and stream is None and (score is not None or not want_score):
        native, lib = _marshal()
        if native is not None and _done(native.decode_top1(lib, preds, mask, alpha, beta, S, sign_mode, top1, score, status)):
            return top1, score, status
    import torch
    K, ap = _nodes(alpha)
    n_beta, bp = _nodes(beta)
    G, N, C = preds.shape
    if N != n_beta:
        raise ValueError("preds.shape[1] must equal len(beta)")
    if top1 is None:
        top1 = torch.full((G, K), -1, dtype=torch.int32, device=preds.device)
    if score is None and want_score:
        score = torch.zeros((G, K), dtype=torch.float32, device=preds.device)
    if status is None:
        status = torch.full((G,), -1, dtype=torch.int32, device=preds.device)
    _check(_entry().approxifer_decode_top1(_dev(preds, torch.float32), _dev(mask, torch.uint8, (G, N)),
                                           _dev(top1, torch.int32, (G, K)),
                                           _dev(score, torch.float32, (G, K)) if score is not None else None,
                                           _dev(status, torch.int32, (G,)), G, K, N, int(S), C, ap, bp, int(sign_mode),
                                           _stream_handle(stream)))
    return top1, score, status


def approxifer_workspace_bytes(G: int, K: int, N: int, S: int, A: int, C: int) -> int:
    """Bytes of device scratch memory with which the Byzantine decoders run fastest at this shape (0: none needed)."""
    return int(load().approxifer_workspace_bytes(int(G), int(K), int(N), int(S), int(A), int(C)))


NO_WORKSPACE = object()


def _decode_byzantine(entry, preds, mask, alpha, beta, S, A, sign_mode, out, adv, status, stream, workspace):
    if out is not None and adv is not None and status is not None and workspace is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.byzantine(lib, entry == "approxifer_decode_byzantine_homogeneous", preds, mask,
                                                         alpha, beta, S, A, sign_mode, out, adv, status,
                                                         None if workspace is NO_WORKSPACE else workspace)):
            return out, adv, status
    import torch
    K, ap = _nodes(alpha)
    n_beta, bp = _nodes(beta)
    G, N, C = preds.shape
    if N != n_beta:
        raise ValueError("preds.shape[1] must equal len(beta)")
    if out is None:
        out = torch.zeros((G, K, C), dtype=torch.float32, device=preds.device)
    if adv is None:
        adv = torch.full((G, max(int(A), 0)), -1, dtype=torch.int32, device=preds.device)
    if status is None:
        status = torch.full((G,), -1, dtype=torch.int32, device=preds.device)
    if workspace is None:
        # the caller left the workspace to the binding: a buffer of the size the library asks for
        need = approxifer_workspace_bytes(G, K, N, S, A, C)
        workspace = torch.empty((need,), dtype=torch.uint8, device=preds.device) if need else NO_WORKSPACE
    if workspace is NO_WORKSPACE:
        ws_ptr, ws_bytes = None, 0
    else:
        if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or not workspace.is_contiguous():
            raise TypeError("workspace must be a contiguous tensor in device memory")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(getattr(_entry(), entry)(_dev(preds, torch.float32), _dev(mask, torch.uint8, (G, N)),
                                    _dev(out, torch.float32, (G, K, C)), _dev(adv, torch.int32, (G, int(A))),
                                    _dev(status, torch.int32, (G,)), G, K, N, int(S), int(A), C, ap, bp,
                                    int(sign_mode), ws_ptr, ws_bytes,
                                    _stream_handle(stream)))
    return out, adv, status


def approxifer_decode_byzantine(preds, mask, alpha, beta, S, A, sign_mode=SIGN_WORKER_INDEX, out=None, adv=None,
                                status=None, stream=None, workspace=None):
    """As approxifer_decode, after locating and dropping A adversaries per group.
    Returns (out [G, K, C] float32, adv [G, A] int32 ascending, status [G] int32).
    workspace: a device tensor (any dtype) passed as the C ABI's d_workspace / workspace_bytes; None allocates
    approxifer_workspace_bytes() bytes for this call; NO_WORKSPACE passes NULL / 0."""
    return _decode_byzantine("approxifer_decode_byzantine", preds, mask, alpha, beta, S, A, sign_mode, out, adv,
                             status, stream, workspace)


def approxifer_decode_byzantine_homogeneous(preds, mask, alpha, beta, S, A, sign_mode=SIGN_WORKER_INDEX, out=None,
                                            adv=None, status=None, stream=None, workspace=None):
    """As approxifer_decode_byzantine, with Algorithm 1's homogeneous fit as the per-class locator."""
    return _decode_byzantine("approxifer_decode_byzantine_homogeneous", preds, mask, alpha, beta, S, A, sign_mode,
                             out, adv, status, stream, workspace)


def approxifer_decode_rational(preds, mask, alpha, beta, S, A, out=None, status=None, stream=None):
    """Algorithm 3: out[g, j, c] = P(alpha_j) / Q(alpha_j) with (P, Q) Algorithm 2's fit per class.
    Returns (out [G, K, C] float32, status [G] int32)."""
    import torch
    K, ap = _nodes(alpha)
    n_beta, bp = _nodes(beta)
    G, N, C = preds.shape
    if N != n_beta:
        raise ValueError("preds.shape[1] must equal len(beta)")
    if out is None:
        out = torch.zeros((G, K, C), dtype=torch.float32, device=preds.device)
    if status is None:
        status = torch.full((G,), -1, dtype=torch.int32, device=preds.device)
    _check(_entry().approxifer_decode_rational(_dev(preds, torch.float32), _dev(mask, torch.uint8, (G, N)),
                                               _dev(out, torch.float32, (G, K, C)), _dev(status, torch.int32, (G,)),
                                               G, K, N, int(S), int(A), C, ap, bp, _stream_handle(stream)))
    return out, status


def approxifer_top1(values, top1=None, score=None, stream=None, want_score=True):
    """values [..., C] float32 device tensor -> (top1 [...] int32, score [...] float32 or None)."""
    if top1 is not None and stream is None and (score is not None or not want_score):
        native, lib = _marshal()
        if native is not None and _done(native.top1(lib, values, top1, score)):
            return top1, score
    import torch
    C = values.shape[-1]
    lead = tuple(values.shape[:-1])
    rows = int(np.prod(lead)) if lead else 1
    if top1 is None:
        top1 = torch.full(lead, -1, dtype=torch.int32, device=values.device)
    if score is None and want_score:
        score = torch.zeros(lead, dtype=torch.float32, device=values.device)
    _check(_entry().approxifer_top1(_dev(values, torch.float32), _dev(top1, torch.int32, lead),
                                    _dev(score, torch.float32, lead) if score is not None else None, rows, C,
                                    _stream_handle(stream)))
    return top1, score


STATIC_WORKSPACE_BYTES = 65536


def approxifer_decode_byzantine_static(preds, mask, alpha, beta, S, A, out, adv, status, sign_mode=SIGN_WORKER_INDEX,
                                       stream=None):
    """approxifer_decode_byzantine on the library's built-in workspace.  Allocates nothing: every output is the
    caller's.  Raises ApproxiferError(-8) for shapes whose workspace exceeds STATIC_WORKSPACE_BYTES."""
    import torch
    K, ap = _nodes(alpha)
    n_beta, bp = _nodes(beta)
    G, N, C = preds.shape
    if N != n_beta:
        raise ValueError("preds.shape[1] must equal len(beta)")
    _check(_entry().approxifer_decode_byzantine_static(_dev(preds, torch.float32), _dev(mask, torch.uint8, (G, N)),
                                                       _dev(out, torch.float32, (G, K, C)),
                                                       _dev(adv, torch.int32, (G, int(A))),
                                                       _dev(status, torch.int32, (G,)), G, K, N, int(S), int(A), C, ap, bp,
                                                       int(sign_mode), _stream_handle(stream)))
    return out, adv, status


def approxifer_wait_mask(arrival, wait_for, mask=None, count=None, stream=None):
    """arrival [G, N] float32 device tensor -> (mask [G, N] uint8, count [G] int32): the wait_for fastest workers."""
    if mask is not None and count is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.wait_mask(lib, arrival, wait_for, mask, count)):
            return mask, count
    import torch
    G, N = arrival.shape
    if mask is None:
        mask = torch.zeros((G, N), dtype=torch.uint8, device=arrival.device)
    if count is None:
        count = torch.full((G,), -1, dtype=torch.int32, device=arrival.device)
    _check(_entry().approxifer_wait_mask(_dev(arrival, torch.float32), _dev(mask, torch.uint8, (G, N)),
                                         _dev(count, torch.int32, (G,)), G, N, int(wait_for),
                                         _stream_handle(stream)))
    return mask, count


# ---- sequences in pages -------------------------------------------------------------------------------------------------
def approxifer_rotary_frequencies(pairs: int, base: float = 10000.0):
    """float64 numpy array [pairs]: base ** (-i / pairs), radians per position."""
    freq = np.empty(max(int(pairs), 0), dtype=np.float64)
    _check(load().approxifer_rotary_frequencies(int(pairs), float(base), freq.ctypes.data_as(ctypes.POINTER(ctypes.c_double))))
    return freq


def _on(stream):
    """Makes a call's stream the current one, so that what is allocated or filled for the call is ordered with it."""
    import contextlib

    import torch
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))


def _dtype_code(dtype) -> int:
    import torch
    codes = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
    if dtype not in codes:
        raise TypeError("expected float32, float16 or bfloat16, got %s" % dtype)
    return codes[dtype]


def _rows(t, dtype):
    """(address, elements between tokens) of a [T, heads, Dh] device tensor whose tokens are contiguous, at any distance."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("expected a tensor in device memory")
    if t.dtype != dtype or t.dim() != 3:
        raise TypeError("expected a %s tensor of three dimensions, got %s of %d" % (dtype, t.dtype, t.dim()))
    T, H, D = t.shape
    if T and ((D > 1 and t.stride(2) != 1) or (H > 1 and t.stride(1) != D)):
        raise TypeError("the heads of a token must be contiguous")
    return t.data_ptr(), t.stride(0) if T > 1 else H * D


def _pools(k_pool, v_pool, dtype, kv=None, Dh=None):
    import torch
    if not isinstance(k_pool, torch.Tensor) or k_pool.dim() != 4:
        raise TypeError("a pool is a tensor [P, Hkv, page, Dh]")
    if (kv is not None and k_pool.shape[1] != kv) or (Dh is not None and k_pool.shape[3] != Dh):
        raise ValueError("the pool's heads do not fit: %s" % (tuple(k_pool.shape),))
    return _dev(k_pool, dtype), _dev(v_pool, dtype, k_pool.shape)


def _sequences(table, lens, starts, T, pool):
    import torch
    B, M = table.shape
    return _Sequences(_dev(table, torch.int32), _dev(lens, torch.int32, (B,)), _dev(starts, torch.int32, (B + 1,)), T, B, M,
                      pool.shape[0], pool.shape[2])


def approxifer_append(q, k, v, k_pool, v_pool, table, lens, starts, freq, q_weight=None, k_weight=None, eps=1e-6, positions=None,
                      axis=None, interleaved=False, q_out=None, status=None, stream=None):
    """Norms (with q_weight, k_weight [Dh]) and rotates the heads of T new tokens' queries and keys and writes keys and values
    into their pages.  q [T, Hq, Dh], k and v [T, Hkv, Dh] (slices of one projection's output will do), pools [P, Hkv, page,
    Dh], table [B, M], lens [B] and starts [B + 1] int32, freq [pairs] float64 on the host; positions [T, axes] int32 and
    axis [pairs] int32 on the host, or None: places in the sequence.  Returns (q_out [T, Hq, Dh], status [B] int32)."""
    if q_out is not None and status is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.append(lib, q, k, v, k_pool, v_pool, table, lens, starts, freq, q_weight, k_weight,
                                                      eps, positions, axis, interleaved, q_out, status)):
            return q_out, status
    import torch
    dtype = k_pool.dtype
    code = _dtype_code(dtype)
    T, Hq, Dh = q.shape
    Hkv = k_pool.shape[1]
    if tuple(k.shape) != (T, Hkv, Dh) or tuple(v.shape) != (T, Hkv, Dh):
        raise ValueError("k and v must be [T, Hkv, Dh] = %s" % ((T, Hkv, Dh),))
    kp, vp = _pools(k_pool, v_pool, dtype, Hkv, Dh)
    qp, q_stride = _rows(q, dtype)
    kk, k_stride = _rows(k, dtype)
    vv, v_stride = _rows(v, dtype)
    with _on(stream):
        if q_out is None:
            q_out = torch.empty((T, Hq, Dh), dtype=dtype, device=q.device)
        if status is None:
            status = torch.full((table.shape[0],), -1, dtype=torch.int32, device=q.device)
    seq = _sequences(table, lens, starts, T, k_pool)
    pairs, fp = _nodes(freq)
    axes = 1
    if positions is not None:
        axes = positions.shape[1] if positions.dim() == 2 else 1
    ap = None
    if axis is not None:
        a = np.ascontiguousarray(axis, dtype=np.int32)
        if a.shape != (pairs,):
            raise ValueError("axis must have one entry for each frequency")
        ap = a.tobytes()
    _check(_entry().approxifer_append(
        ctypes.byref(seq), Hq, Hkv, Dh, code, qp, q_stride, kk, k_stride, vv, v_stride, _dev(q_out, dtype, (T, Hq, Dh)), kp, vp,
        _dev(q_weight, dtype, (Dh,)) if q_weight is not None else None,
        _dev(k_weight, dtype, (Dh,)) if k_weight is not None else None, float(eps),
        _dev(positions, torch.int32, (T, axes) if positions.dim() == 2 else (T,)) if positions is not None else None, axes, fp, ap,
        pairs, int(bool(interleaved)), _dev(status, torch.int32, (table.shape[0],)), _stream_handle(stream)))
    return q_out, status


def approxifer_attend_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window=0, sinks=0) -> int:
    """Bytes of scratch memory with which approxifer_attend is fastest (0: none); dtype a torch dtype."""
    return int(load().approxifer_attend_workspace_bytes(int(T), int(B), int(Hq), int(Hkv), int(Dh), _dtype_code(dtype), int(max_rows),
                                                        int(max_len), int(window), int(sinks)))


def _scratch(workspace):
    import torch
    if workspace is NO_WORKSPACE:
        return None, 0
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor in device memory")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def approxifer_attend(q, k_pool, v_pool, table, lens, starts, max_rows, max_len, window=0, sinks=0, scale=None, out=None,
                      status=None, workspace=None, stream=None):
    """Causal attention of T new tokens (already appended) to their sequences: q [T, Hq, Dh], the rest as approxifer_append;
    max_rows and max_len bound the sequences' new tokens and lengths.  window (0: none) and sinks limit what a token sees,
    scale defaults to Dh ** -0.5.  workspace as approxifer_decode_byzantine's, of approxifer_attend_workspace_bytes().
    Returns (out [T, Hq, Dh], status [B] int32)."""
    if out is not None and status is not None and workspace is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.attend(lib, q, k_pool, v_pool, table, lens, starts, max_rows, max_len, window, sinks,
                                                      scale, out, status, None if workspace is NO_WORKSPACE else workspace)):
            return out, status
    import torch
    dtype = k_pool.dtype
    code = _dtype_code(dtype)
    T, Hq, Dh = q.shape
    Hkv = k_pool.shape[1]
    kp, vp = _pools(k_pool, v_pool, dtype, None, Dh)
    qp, q_stride = _rows(q, dtype)
    with _on(stream):
        if out is None:
            out = torch.empty((T, Hq, Dh), dtype=dtype, device=q.device)
        if status is None:
            status = torch.full((table.shape[0],), -1, dtype=torch.int32, device=q.device)
        if workspace is None:
            need = approxifer_attend_workspace_bytes(T, table.shape[0], Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks)
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device) if need else NO_WORKSPACE
    ws_ptr, ws_bytes = _scratch(workspace)
    seq = _sequences(table, lens, starts, T, k_pool)
    _check(_entry().approxifer_attend(
        ctypes.byref(seq), Hq, Hkv, Dh, code, qp, q_stride, kp, vp, _dev(out, dtype, (T, Hq, Dh)), int(max_rows), int(max_len),
        int(window), int(sinks), Dh ** -0.5 if scale is None else float(scale), _dev(status, torch.int32, (table.shape[0],)), ws_ptr,
        ws_bytes, _stream_handle(stream)))
    return out, status


def approxifer_attend_shared_workspace_bytes(T, B, C, Hq, Hkv, Dh, dtype, max_rows, max_len, max_shared, window=0, sinks=0) -> int:
    """Bytes of scratch memory with which approxifer_attend_shared is fastest (0: none); dtype a torch dtype."""
    return int(load().approxifer_attend_shared_workspace_bytes(int(T), int(B), int(C), int(Hq), int(Hkv), int(Dh), _dtype_code(dtype),
                                                               int(max_rows), int(max_len), int(max_shared), int(window), int(sinks)))


def approxifer_attend_shared_pays(T, B, C, Hq, Hkv, Dh, dtype, page, max_rows, max_len, max_shared, window=0, sinks=0) -> bool:
    """Whether approxifer_attend_shared is expected to take less time than approxifer_attend; dtype a torch dtype."""
    return bool(load().approxifer_attend_shared_pays(int(T), int(B), int(C), int(Hq), int(Hkv), int(Dh), _dtype_code(dtype), int(page),
                                                     int(max_rows), int(max_len), int(max_shared), int(window), int(sinks)))


def approxifer_attend_shared(q, k_pool, v_pool, table, lens, starts, groups, shared, max_rows, max_len, max_shared, window=0, sinks=0,
                             scale=None, out=None, status=None, workspace=None, stream=None):
    """approxifer_attend for sequences that begin alike: sequences groups[c] .. groups[c + 1] - 1 have their first shared[c] places in common
    (groups [C + 1], shared [C] int32; max_shared bounds the latter), and what they have in common is read once for all of them.
    Returns (out [T, Hq, Dh], status [B] int32)."""
    if out is not None and status is not None and workspace is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.attend_shared(lib, q, k_pool, v_pool, table, lens, starts, groups, shared, max_rows, max_len,
                                                             max_shared, window, sinks, scale, out, status,
                                                             None if workspace is NO_WORKSPACE else workspace)):
            return out, status
    import torch
    dtype = k_pool.dtype
    code = _dtype_code(dtype)
    T, Hq, Dh = q.shape
    Hkv = k_pool.shape[1]
    B = table.shape[0]
    kp, vp = _pools(k_pool, v_pool, dtype, None, Dh)
    qp, q_stride = _rows(q, dtype)
    C = shared.numel()
    gp, sp = _dev(groups, torch.int32, (C + 1,)), _dev(shared, torch.int32, (C,))
    with _on(stream):
        if out is None:
            out = torch.empty((T, Hq, Dh), dtype=dtype, device=q.device)
        if status is None:
            status = torch.full((B,), -1, dtype=torch.int32, device=q.device)
        if workspace is None:
            need = approxifer_attend_shared_workspace_bytes(T, B, C, Hq, Hkv, Dh, dtype, max_rows, max_len, max_shared, window, sinks)
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device) if need else NO_WORKSPACE
    ws_ptr, ws_bytes = _scratch(workspace)
    seq = _sequences(table, lens, starts, T, k_pool)
    _check(_entry().approxifer_attend_shared(
        ctypes.byref(seq), Hq, Hkv, Dh, code, qp, q_stride, kp, vp, _dev(out, dtype, (T, Hq, Dh)), gp, sp, C, int(max_rows), int(max_len),
        int(max_shared), int(window), int(sinks), Dh ** -0.5 if scale is None else float(scale), _dev(status, torch.int32, (B,)), ws_ptr,
        ws_bytes, _stream_handle(stream)))
    return out, status


def approxifer_attend_mass_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window=0, sinks=0) -> int:
    """Bytes of scratch memory with which approxifer_attend_mass is fastest; dtype a torch dtype."""
    return int(load().approxifer_attend_mass_workspace_bytes(int(T), int(B), int(Hq), int(Hkv), int(Dh), _dtype_code(dtype), int(max_rows),
                                                             int(max_len), int(window), int(sinks)))


def approxifer_attend_mass(q, k_pool, v_pool, table, lens, starts, mass, max_rows, max_len, window=0, sinks=0, scale=None, out=None,
                           status=None, workspace=None, stream=None):
    """approxifer_attend, which adds the weights that it gives every place of a sequence to mass [B, L] float32, L at least the sequences'
    length.  workspace: of approxifer_attend_mass_workspace_bytes(), or None.  Returns (out [T, Hq, Dh], status [B] int32)."""
    if out is not None and status is not None and workspace is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.attend_mass(lib, q, k_pool, v_pool, table, lens, starts, mass, max_rows, max_len, window,
                                                           sinks, scale, out, status, None if workspace is NO_WORKSPACE else workspace)):
            return out, status
    import torch
    dtype = k_pool.dtype
    code = _dtype_code(dtype)
    T, Hq, Dh = q.shape
    Hkv = k_pool.shape[1]
    B = table.shape[0]
    kp, vp = _pools(k_pool, v_pool, dtype, None, Dh)
    qp, q_stride = _rows(q, dtype)
    if not isinstance(mass, torch.Tensor) or mass.dim() != 2:
        raise TypeError("mass is a tensor [B, L]")
    with _on(stream):
        if out is None:
            out = torch.empty((T, Hq, Dh), dtype=dtype, device=q.device)
        if status is None:
            status = torch.full((B,), -1, dtype=torch.int32, device=q.device)
        if workspace is None:
            need = approxifer_attend_mass_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks)
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device) if need else NO_WORKSPACE
    ws_ptr, ws_bytes = _scratch(workspace)
    seq = _sequences(table, lens, starts, T, k_pool)
    _check(_entry().approxifer_attend_mass(
        ctypes.byref(seq), Hq, Hkv, Dh, code, qp, q_stride, kp, vp, _dev(out, dtype, (T, Hq, Dh)),
        _dev(mass, torch.float32, (B, mass.shape[1])), mass.shape[1], int(max_rows), int(max_len), int(window), int(sinks),
        Dh ** -0.5 if scale is None else float(scale), _dev(status, torch.int32, (B,)), ws_ptr, ws_bytes, _stream_handle(stream)))
    return out, status


def approxifer_cache_reserve(table, lens, refs, add, page, status=None, stream=None):
    """Room for add[b] more tokens of every sequence, in place: table [B, M], lens [B], refs [P], add [B] int32.
    Returns status [B] int32."""
    if status is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.cache_reserve(lib, table, lens, refs, add, page, status)):
            return status
    import torch
    B, M = table.shape
    with _on(stream):
        if status is None:
            status = torch.full((B,), -1, dtype=torch.int32, device=table.device)
    _check(_entry().approxifer_cache_reserve(_dev(table, torch.int32), _dev(lens, torch.int32, (B,)), _dev(refs, torch.int32),
                                             _dev(add, torch.int32, (B,)), _dev(status, torch.int32, (B,)), B, M, refs.numel(),
                                             int(page), _stream_handle(stream)))
    return status


def approxifer_cache_workspace_bytes(B: int, B_out: int, P: int) -> int:
    """Bytes of scratch memory that approxifer_cache_fork and approxifer_cache_compact need."""
    return int(load().approxifer_cache_workspace_bytes(int(B), int(B_out), int(P)))


def _planes(pools, P):
    """(address, planes, bytes of a page, tokens of a page) of pools [.., P, Hkv, page, Dh]."""
    import torch
    if not isinstance(pools, torch.Tensor) or not pools.is_cuda or not pools.is_contiguous() or pools.dim() < 4:
        raise TypeError("pools must be a contiguous tensor [.., P, Hkv, page, Dh] in device memory")
    if pools.shape[-4] != P:
        raise ValueError("the pools have %d pages, refs %d" % (pools.shape[-4], P))
    page_bytes = pools.shape[-3] * pools.shape[-2] * pools.shape[-1] * pools.element_size()
    return pools.data_ptr(), pools.shape[:-4].numel(), page_bytes, pools.shape[-2]


def approxifer_cache_fork(pools, table, lens, refs, parents, keep=None, table_out=None, lens_out=None, refs_out=None, status=None,
                          workspace=None, stream=None):
    """New sequences out of old ones: sequence i continues old sequence parents[i] (-1: empty), all of it or keep[i] tokens.
    pools [.., P, Hkv, page, Dh] hold all layers' keys and values; table [B, M], lens [B], refs [P], parents and keep [B_out]
    int32.  Returns (table_out [B_out, M], lens_out [B_out], refs_out [P], status [B_out])."""
    if (table_out is not None and lens_out is not None and refs_out is not None and status is not None and workspace is not None
            and stream is None):
        native, lib = _marshal()
        if native is not None and _done(native.cache_fork(lib, pools, table, lens, refs, parents, keep, table_out, lens_out, refs_out,
                                                          status, workspace)):
            return table_out, lens_out, refs_out, status
    import torch
    i32 = torch.int32
    B, M = table.shape
    P, n = refs.numel(), parents.numel()
    at, planes, page_bytes, page = _planes(pools, P)
    with _on(stream):
        if table_out is None:
            table_out = torch.empty((n, M), dtype=i32, device=table.device)
        if lens_out is None:
            lens_out = torch.empty((n,), dtype=i32, device=table.device)
        if refs_out is None:
            refs_out = torch.empty((P,), dtype=i32, device=table.device)
        if status is None:
            status = torch.full((n,), -1, dtype=i32, device=table.device)
        if workspace is None:
            workspace = torch.empty((approxifer_cache_workspace_bytes(B, n, P),), dtype=torch.uint8, device=table.device)
    ws_ptr, ws_bytes = _scratch(workspace)
    _check(_entry().approxifer_cache_fork(
        _dev(table, i32), _dev(lens, i32, (B,)), _dev(refs, i32), _dev(parents, i32, (n,)),
        _dev(keep, i32, (n,)) if keep is not None else None, _dev(table_out, i32, (n, M)), _dev(lens_out, i32, (n,)),
        _dev(refs_out, i32, (P,)), _dev(status, i32, (n,)), at, planes, page_bytes, B, n, M, P, page, ws_ptr, ws_bytes,
        _stream_handle(stream)))
    return table_out, lens_out, refs_out, status


def approxifer_cache_compact(pools, table, lens, refs, moved=None, live=None, workspace=None, stream=None):
    """Moves the live pages of all pools together, in place; table and refs follow.  Returns (moved [P] int32: where each page
    is now, -1 for free ones; live [1] int32)."""
    if moved is not None and live is not None and workspace is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.cache_compact(lib, pools, table, lens, refs, moved, live, workspace)):
            return moved, live
    import torch
    i32 = torch.int32
    B, M = table.shape
    P = refs.numel()
    at, planes, page_bytes, page = _planes(pools, P)
    with _on(stream):
        if moved is None:
            moved = torch.empty((P,), dtype=i32, device=table.device)
        if live is None:
            live = torch.empty((1,), dtype=i32, device=table.device)
        if workspace is None:
            workspace = torch.empty((approxifer_cache_workspace_bytes(B, B, P),), dtype=torch.uint8, device=table.device)
    ws_ptr, ws_bytes = _scratch(workspace)
    _check(_entry().approxifer_cache_compact(
        _dev(table, i32), _dev(lens, i32, (B,)), _dev(refs, i32), _dev(moved, i32, (P,)), _dev(live, i32, (1,)), at, planes,
        page_bytes, B, M, P, page, ws_ptr, ws_bytes, _stream_handle(stream)))
    return moved, live


def approxifer_cache_evict_workspace_bytes(B: int, budget: int, P: int, page: int) -> int:
    """Bytes of scratch memory that approxifer_cache_evict needs."""
    return int(load().approxifer_cache_evict_workspace_bytes(int(B), int(budget), int(P), int(page)))


def approxifer_cache_evict(pools, table, lens, refs, mass, budget, first=0, recent=0, kept=None, status=None, workspace=None,
                           stream=None):
    """Cuts every sequence of more than `budget` tokens to that many, in place: its `first` first and `recent` last ones and those of the
    largest mass between them, in their order.  pools [.., P, Hkv, page, Dh] hold all layers' keys and values; table [B, M], lens
    [B], refs [P] int32, mass [B, L] float32.  Returns (kept [B, budget] int32: the places that stay, then -1; status [B] int32)."""
    if kept is not None and status is not None and workspace is not None and stream is None:
        native, lib = _marshal()
        if native is not None and _done(native.cache_evict(lib, pools, table, lens, refs, mass, budget, first, recent, kept, status,
                                                           workspace)):
            return kept, status
    import torch
    i32 = torch.int32
    B, M = table.shape
    P, budget = refs.numel(), int(budget)
    at, planes, _, page = _planes(pools, P)
    if not isinstance(mass, torch.Tensor) or mass.dim() != 2:
        raise TypeError("mass is a tensor [B, L]")
    with _on(stream):
        if kept is None:
            kept = torch.empty((B, max(budget, 0)), dtype=i32, device=table.device)
        if status is None:
            status = torch.full((B,), -1, dtype=i32, device=table.device)
        if workspace is None:
            workspace = torch.empty((approxifer_cache_evict_workspace_bytes(B, budget, P, page),), dtype=torch.uint8, device=table.device)
    ws_ptr, ws_bytes = _scratch(workspace)
    _check(_entry().approxifer_cache_evict(
        _dev(table, i32), _dev(lens, i32, (B,)), _dev(refs, i32), _dev(mass, torch.float32, (B, mass.shape[1])), mass.shape[1],
        _dev(kept, i32, (B, max(budget, 0))), _dev(status, i32, (B,)), at, planes, pools.shape[-3],
        pools.shape[-1] * pools.element_size(), B, M, P, page, budget, int(first), int(recent), ws_ptr, ws_bytes,
        _stream_handle(stream)))
    return kept, status
