"""Python binding of libsplitee.so, the MI355X DP-masked linear layer.

Argument marshalling only: every function below forwards to the C entry point
of the same name (declared in include/splitee.h) with device pointers taken
from torch tensors and the current torch stream.  All arithmetic runs in the
HIP kernels; there is no fallback.  If the library is not built the import
still works but every call raises.
"""
import ctypes
import os
import typing

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsplitee.so")

SPLITEE_OK = 0
SPLITEE_MECH_LAPLACE, SPLITEE_MECH_GAUSSIAN, SPLITEE_MECH_NONE = 0, 1, 2
SPLITEE_F32, SPLITEE_BF16, SPLITEE_BF16_TILED = 0, 1, 2
SPLITEE_PREC_F32, SPLITEE_PREC_BF16, SPLITEE_PREC_BF16X3 = 0, 1, 2
MECHS = {"laplace": SPLITEE_MECH_LAPLACE, "gaussian": SPLITEE_MECH_GAUSSIAN, "none": SPLITEE_MECH_NONE}
PRECS = {"f32": SPLITEE_PREC_F32, "bf16": SPLITEE_PREC_BF16, "bf16x3": SPLITEE_PREC_BF16X3}
SPLITEE_BOUND_LN, SPLITEE_BOUND_ATT, SPLITEE_BOUND_ACT = 0, 1, 2

EXPORTED = [
    "splitee_abi_version", "splitee_status_string", "splitee_noise_gen", "splitee_mask",
    "splitee_masked_linear", "splitee_unmask", "splitee_fused_workspace_bytes",
    "splitee_masked_linear_fused", "splitee_correction",
    "splitee_noise_mask", "splitee_gemm_workspace_bytes", "splitee_masked_linear_unmask",
    "splitee_noise_gen_multi", "splitee_spectral_norm_workspace_bytes", "splitee_spectral_norm",
    "splitee_sensitivity_workspace_bytes", "splitee_sensitivity", "splitee_eps_per_token",
    "splitee_bank_path", "splitee_bank_workspace_bytes", "splitee_bank_create", "splitee_bank_open",
    "splitee_bank_info", "splitee_bank_load", "splitee_bank_close",
    "splitee_f64_workspace_bytes", "splitee_masked_linear_fused_f64", "splitee_correction_f64",
    "splitee_tiled_weights_bytes", "splitee_tile_weights", "splitee_masked_linear_fused_noalloc",
    "splitee_epilogue_workspace_bytes", "splitee_linear_epilogue", "splitee_grouped_linear",
    "splitee_route_workspace_bytes", "splitee_route", "splitee_combine",
]
# test hooks (include/splitee_probe.h)
EXPORTED_PROBE = ["splitee_transform_probe", "splitee_mfma_probe", "splitee_spectral_norm_probe",
                  "splitee_linear_plan_probe"]
SPLITEE_PATH_NONE, SPLITEE_PATH_STREAMED, SPLITEE_PATH_RESIDENT, SPLITEE_PATH_GAVE_UP = 0, 1, 2, 3
SPLITEE_PREC_F64 = 3
SPLITEE_ERR_IO, SPLITEE_ERR_EXHAUSTED, SPLITEE_ERR_FORMAT, SPLITEE_ERR_BUSY = -8, -9, -10, -11
SPLITEE_ERR_SCRATCH = -12
SPLITEE_NOALLOC_SCRATCH_BYTES = 64 << 20
SPLITEE_ACT_NONE, SPLITEE_ACT_SILU, SPLITEE_ACT_GELU, SPLITEE_ACT_GELU_TANH, SPLITEE_ACT_RELU = 0, 1, 2, 3, 4
ACTS = {"none": SPLITEE_ACT_NONE, "silu": SPLITEE_ACT_SILU, "gelu": SPLITEE_ACT_GELU,
        "gelu_tanh": SPLITEE_ACT_GELU_TANH, "relu": SPLITEE_ACT_RELU}
SPLITEE_SCORE_SOFTMAX, SPLITEE_SCORE_SIGMOID = 0, 1
SCORES = {"softmax": SPLITEE_SCORE_SOFTMAX, "sigmoid": SPLITEE_SCORE_SIGMOID}


class BankInfo(ctypes.Structure):
    """splitee_bank_info_t"""
    _fields_ = [("K", ctypes.c_int64), ("N", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("stream_id", ctypes.c_uint64), ("mech", ctypes.c_int32), ("prec", ctypes.c_int32),
                ("sensitivity", ctypes.c_double), ("epsilon", ctypes.c_double), ("row0", ctypes.c_int64),
                ("rows", ctypes.c_int64), ("consumed", ctypes.c_int64), ("bytes_stored", ctypes.c_int64),
                ("bytes_with_masks", ctypes.c_int64)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class Epilogue(ctypes.Structure):
    """splitee_epilogue_t"""
    _fields_ = [("C", ctypes.c_void_p), ("ldc", ctypes.c_int64), ("bias", ctypes.c_void_p),
                ("bias_stride", ctypes.c_int64), ("residual", ctypes.c_void_p), ("ldres", ctypes.c_int64),
                ("act", ctypes.c_int32), ("gated", ctypes.c_int32), ("out_type", ctypes.c_int32)]


class SpliteeError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (fn, _status_text(status), status))


_lib = None


def load():
    """Load libsplitee.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libsplitee.so is not built (run __graft_entry__.build())")
    lib = ctypes.CDLL(LIB_PATH)
    P, I, I64, U64, D, SZ = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64,
                             ctypes.c_double, ctypes.c_size_t)
    sig = {
        "splitee_abi_version": (I, []),
        "splitee_status_string": (ctypes.c_char_p, [I]),
        "splitee_noise_gen": (I, [P, I64, I64, I64, I, D, D, U64, U64, U64, P]),
        "splitee_mask": (I, [P, I64, P, I64, P, I, I64, I64, I64, P]),
        "splitee_masked_linear": (I, [P, I, I64, P, I, I64, P, I64, I64, I64, I64, P]),
        "splitee_unmask": (I, [P, I64, P, I64, P, I64, I64, I64, P]),
        "splitee_fused_workspace_bytes": (SZ, [I64, I64, I64, I]),
        "splitee_masked_linear_fused": (I, [P, I64, P, I, I64, P, I64, P, I64, I64, I64, I64, I, D, D,
                                            U64, U64, U64, P, I, P, SZ, P]),
        "splitee_correction": (I, [P, I64, P, I, I64, I64, I64, I64, I, D, D, U64, U64, U64, I, P, SZ,
                                   P]),
        "splitee_transform_probe": (I, [P, I64, I, I, P, P]),
        "splitee_noise_mask": (I, [P, I64, P, I, I64, I64, I64, I, D, D, U64, U64, U64, P]),
        "splitee_gemm_workspace_bytes": (SZ, [I64, I64, I64, I]),
        "splitee_masked_linear_unmask": (I, [P, I, I64, P, I, I64, P, I64, P, I64, I64, I64, I64, P,
                                             SZ, P]),
        "splitee_noise_gen_multi": (I, [P, P, P, P, I, I, P, U64, I64, I, D, D, U64, U64, P]),
        "splitee_spectral_norm_workspace_bytes": (SZ, [I64, I64, I]),
        "splitee_spectral_norm": (I, [P, I, I64, I64, I64, I, U64, U64, P, P, P, SZ, P]),
        "splitee_sensitivity_workspace_bytes": (SZ, []),
        "splitee_sensitivity": (I, [I, I64, P, P, D, D, P, P, SZ, P]),
        "splitee_eps_per_token": (I, [D, I64, P]),
        "splitee_bank_path": (I, [ctypes.c_char_p, I64, I64, U64, ctypes.c_char_p, SZ]),
        "splitee_bank_workspace_bytes": (SZ, [I64, I64, I]),
        "splitee_bank_create": (I, [ctypes.c_char_p, P, I, I64, I64, I64, I, D, D, U64, U64, U64, I64, I, P, SZ,
                                    P]),
        "splitee_bank_open": (I, [ctypes.c_char_p, ctypes.POINTER(ctypes.c_void_p)]),
        "splitee_bank_info": (I, [P, ctypes.POINTER(BankInfo)]),
        "splitee_bank_load": (I, [P, I64, P, I64, I, ctypes.POINTER(ctypes.c_int64), P]),
        "splitee_bank_close": (I, [P]),
        "splitee_f64_workspace_bytes": (SZ, [I64, I64, I64]),
        "splitee_masked_linear_fused_f64": (I, [P, I64, P, I, I64, P, I64, P, I64, I64, I64, I64, I, D, D, U64,
                                                U64, U64, P, SZ, P]),
        "splitee_correction_f64": (I, [P, I64, P, I, I64, I64, I64, I64, I, D, D, U64, U64, U64, P, SZ, P]),
        "splitee_tiled_weights_bytes": (SZ, [I64, I64]),
        "splitee_tile_weights": (I, [P, I64, I64, I64, P, P]),
        "splitee_mfma_probe": (I, [I, I, P, P, D, P, P]),
        "splitee_spectral_norm_probe": (I, [P, I, I64, I64, I64, I, U64, U64, P, P, P, SZ, I64, P, P]),
        "splitee_masked_linear_fused_noalloc": (I, [P, I64, P, I, I64, P, I64, P, I64, I64, I64, I64, I, D, D,
                                                    U64, U64, U64, P, I, P]),
        "splitee_linear_plan_probe": (I, [I64, I64, I, I64, I64, I, I, P]),
        "splitee_epilogue_workspace_bytes": (SZ, [I64, I64, I64, I, I]),
        "splitee_linear_epilogue": (I, [P, I, I64, P, I, I64, P, P, I64, I64, I64, I64, P, SZ, P]),
        "splitee_grouped_linear": (I, [P, I, I64, I64, P, P, I64, P, I, I64, I64, P, P, I64, I64, I64, I64, P]),
        "splitee_route_workspace_bytes": (SZ, [I64, I64, I64]),
        "splitee_route": (I, [P, I64, I64, I64, I64, I, I, P, P, P, P, P, P, SZ, P]),
        "splitee_combine": (I, [P, I, I64, I64, P, P, P, I64, P, I, I64, I64, I64, I64, P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _status_text(status):
    try:
        return load().splitee_status_string(status).decode()
    except Exception:  # library missing
        return "status"


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # the handle alone: torch.cuda.current_stream() builds a Stream object around it, 2.8 us a
        # call against 0.3 (of 12.5 us of host time of a small fused call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return stream


def _check(fn, status):
    if status != SPLITEE_OK:
        raise SpliteeError(fn, status)


class TiledWeights:
    """A bfloat16 N x K weight matrix stored in the tiled order of
    splitee_tile_weights (`data`, a flat device tensor; for the experts of grouped_linear
    one row of an experts x elements tensor each).  Passed wherever a W tensor
    is taken; shape, dtype, stride and data_ptr describe the logical matrix."""

    dtype = torch.bfloat16

    def __init__(self, data, N, K):
        self.data, self.N, self.K = data, N, K

    @property
    def shape(self):
        return (self.N, self.K)

    @property
    def device(self):
        return self.data.device

    @property
    def is_cuda(self):
        return self.data.is_cuda

    def stride(self, dim):
        return (self.K, 1)[dim]

    def data_ptr(self):
        return self.data.data_ptr()


def _wtype(W, name="W"):
    """w_type of a weight tensor; any other type would be read as one of these, and past its end."""
    if isinstance(W, TiledWeights):
        if W.data.dtype != torch.bfloat16 and W.data.dtype.is_floating_point:  # (integers hold its bytes)
            raise ValueError("%s: tiled weights are bfloat16, not %s" % (name, W.data.dtype))
        return SPLITEE_BF16_TILED
    if W.dtype == torch.bfloat16:
        return SPLITEE_BF16
    if W.dtype != torch.float32:
        raise ValueError("%s: expected float32 or bfloat16, not %s" % (name, W.dtype))
    return SPLITEE_F32


# ------------------------------------------------------------ C entry points

def splitee_abi_version():
    return load().splitee_abi_version()


def splitee_status_string(status):
    return load().splitee_status_string(status).decode()


def splitee_tiled_weights_bytes(N, K):
    return load().splitee_tiled_weights_bytes(N, K)


def splitee_tile_weights(W, ldw, N, K, Wt, stream=None):
    _check("splitee_tile_weights", load().splitee_tile_weights(_ptr(W), ldw, N, K, _ptr(Wt), _stream(stream)))


def splitee_noise_gen(eta, ld_eta, M, K, mech, sensitivity, epsilon, seed, stream_id, row0=0,
                      stream=None):
    _check("splitee_noise_gen", load().splitee_noise_gen(
        _ptr(eta), ld_eta, M, K, mech, sensitivity, epsilon, seed, stream_id, row0, _stream(stream)))


def splitee_noise_gen_multi(etas, ld_etas, Ks, stream_ids, M, mech, sensitivity, epsilon, seed,
                            row0=0, reps=1, rep_strides=None, rep_sid_step=0, stream=None):
    """etas, ld_etas, Ks, stream_ids (and rep_strides when reps > 1): sequences of
    equal length, one entry per noise block."""
    n = len(etas)
    if not (len(ld_etas) == len(Ks) == len(stream_ids) == n):
        raise ValueError("splitee_noise_gen_multi: per-block sequences differ in length")
    ptrs = (ctypes.c_void_p * max(n, 1))(*[_ptr(e) for e in etas])
    lds = (ctypes.c_int64 * max(n, 1))(*ld_etas)
    ks = (ctypes.c_int64 * max(n, 1))(*Ks)
    sids = (ctypes.c_uint64 * max(n, 1))(*stream_ids)
    strides = None
    if rep_strides is not None:
        if len(rep_strides) != n:
            raise ValueError("splitee_noise_gen_multi: rep_strides differs in length")
        strides = ctypes.cast((ctypes.c_int64 * max(n, 1))(*rep_strides), ctypes.c_void_p)
    _check("splitee_noise_gen_multi", load().splitee_noise_gen_multi(
        ctypes.cast(ptrs, ctypes.c_void_p), ctypes.cast(lds, ctypes.c_void_p), ctypes.cast(ks, ctypes.c_void_p),
        ctypes.cast(sids, ctypes.c_void_p), n, reps, strides, rep_sid_step, M, mech, sensitivity, epsilon,
        seed, row0, _stream(stream)))


def splitee_mask(X, ldx, eta, ld_eta, Xt, out_prec, ldxt, M, K, stream=None):
    _check("splitee_mask", load().splitee_mask(
        _ptr(X), ldx, _ptr(eta), ld_eta, _ptr(Xt), out_prec, ldxt, M, K, _stream(stream)))


def splitee_masked_linear(Xt, in_prec, ldxt, W, w_type, ldw, R, ldr, M, N, K, stream=None):
    _check("splitee_masked_linear", load().splitee_masked_linear(
        _ptr(Xt), in_prec, ldxt, _ptr(W), w_type, ldw, _ptr(R), ldr, M, N, K, _stream(stream)))


def splitee_unmask(R, ldr, C, ldc, Y, ldy, M, N, stream=None):
    _check("splitee_unmask", load().splitee_unmask(
        _ptr(R), ldr, _ptr(C), ldc, _ptr(Y), ldy, M, N, _stream(stream)))


def splitee_fused_workspace_bytes(M, N, K, prec):
    return load().splitee_fused_workspace_bytes(M, N, K, prec)


def splitee_masked_linear_fused(X, ldx, W, w_type, ldw, C, ldc, Y, ldy, M, N, K, mech, sensitivity,
                                epsilon, seed, stream_id, row0, eta_override, prec, workspace,
                                workspace_bytes, stream=None):
    _check("splitee_masked_linear_fused", load().splitee_masked_linear_fused(
        _ptr(X), ldx, _ptr(W), w_type, ldw, _ptr(C), ldc, _ptr(Y), ldy, M, N, K, mech, sensitivity,
        epsilon, seed, stream_id, row0, _ptr(eta_override), prec, _ptr(workspace), workspace_bytes,
        _stream(stream)))


def splitee_masked_linear_fused_noalloc(X, ldx, W, w_type, ldw, C, ldc, Y, ldy, M, N, K, mech, sensitivity,
                                        epsilon, seed, stream_id, row0, eta_override, prec, stream=None):
    _check("splitee_masked_linear_fused_noalloc", load().splitee_masked_linear_fused_noalloc(
        _ptr(X), ldx, _ptr(W), w_type, ldw, _ptr(C), ldc, _ptr(Y), ldy, M, N, K, mech, sensitivity, epsilon, seed,
        stream_id, row0, _ptr(eta_override), prec, _stream(stream)))


def splitee_correction(C, ldc, W, w_type, ldw, M, N, K, mech, sensitivity, epsilon, seed,
                       stream_id, row0, prec, workspace, workspace_bytes, stream=None):
    _check("splitee_correction", load().splitee_correction(
        _ptr(C), ldc, _ptr(W), w_type, ldw, M, N, K, mech, sensitivity, epsilon, seed, stream_id,
        row0, prec, _ptr(workspace), workspace_bytes, _stream(stream)))


def splitee_transform_probe(words, n, fn, force_slow, out, stream=None):
    _check("splitee_transform_probe", load().splitee_transform_probe(
        _ptr(words), n, fn, force_slow, _ptr(out), _stream(stream)))


def splitee_mfma_probe(op, n, a, b, c, d, stream=None):
    _check("splitee_mfma_probe", load().splitee_mfma_probe(op, n, _ptr(a), _ptr(b), float(c), _ptr(d),
                                                           _stream(stream)))


def splitee_noise_mask(X, ldx, Xt, out_prec, ldxt, M, K, mech, sensitivity, epsilon, seed,
                       stream_id, row0=0, stream=None):
    _check("splitee_noise_mask", load().splitee_noise_mask(
        _ptr(X), ldx, _ptr(Xt), out_prec, ldxt, M, K, mech, sensitivity, epsilon, seed, stream_id,
        row0, _stream(stream)))


def splitee_gemm_workspace_bytes(M, N, K, prec):
    return load().splitee_gemm_workspace_bytes(M, N, K, prec)


def splitee_masked_linear_unmask(Xt, in_prec, ldxt, W, w_type, ldw, C, ldc, Y, ldy, M, N, K,
                                 workspace, workspace_bytes, stream=None):
    _check("splitee_masked_linear_unmask", load().splitee_masked_linear_unmask(
        _ptr(Xt), in_prec, ldxt, _ptr(W), w_type, ldw, _ptr(C), ldc, _ptr(Y), ldy, M, N, K,
        _ptr(workspace), workspace_bytes, _stream(stream)))


def splitee_spectral_norm_workspace_bytes(N, K, iters):
    return load().splitee_spectral_norm_workspace_bytes(N, K, iters)


def splitee_spectral_norm(W, w_type, ldw, N, K, iters, seed, stream_id, workspace, workspace_bytes,
                          history=False, stream=None):
    """Returns sigma of the last round, or (sigma, [sigma of every round]) with history."""
    sigma = ctypes.c_double()
    hist = (ctypes.c_double * iters)() if history and iters > 0 else None
    _check("splitee_spectral_norm", load().splitee_spectral_norm(
        _ptr(W), w_type, ldw, N, K, iters, seed, stream_id, ctypes.byref(sigma),
        ctypes.cast(hist, ctypes.c_void_p) if hist is not None else None, _ptr(workspace), workspace_bytes,
        _stream(stream)))
    return (sigma.value, list(hist) if hist is not None else []) if history else sigma.value


def splitee_spectral_norm_probe(W, w_type, ldw, N, K, iters, seed, stream_id, workspace, workspace_bytes, spins=-1,
                                stream=None):
    """Returns (path, [sigma of every round]); path as splitee_spectral_path."""
    sigma, path, hist = ctypes.c_double(), ctypes.c_int(), (ctypes.c_double * iters)()
    _check("splitee_spectral_norm_probe", load().splitee_spectral_norm_probe(
        _ptr(W), w_type, ldw, N, K, iters, seed, stream_id, ctypes.byref(sigma),
        ctypes.cast(hist, ctypes.c_void_p), _ptr(workspace), workspace_bytes, spins, ctypes.byref(path),
        _stream(stream)))
    return path.value, list(hist)


def splitee_sensitivity_workspace_bytes():
    return load().splitee_sensitivity_workspace_bytes()


def splitee_sensitivity(bound, d, alpha, beta, w_norm_a, w_norm_b, workspace, workspace_bytes, stream=None):
    """Returns the bound Delta f."""
    delta = ctypes.c_double()
    _check("splitee_sensitivity", load().splitee_sensitivity(
        bound, d, _ptr(alpha), _ptr(beta), w_norm_a, w_norm_b, ctypes.byref(delta), _ptr(workspace),
        workspace_bytes, _stream(stream)))
    return delta.value


def splitee_eps_per_token(eps_total, n):
    eps = ctypes.c_double()
    _check("splitee_eps_per_token", load().splitee_eps_per_token(eps_total, n, ctypes.byref(eps)))
    return eps.value


def splitee_f64_workspace_bytes(M, N, K):
    return load().splitee_f64_workspace_bytes(M, N, K)


def splitee_masked_linear_fused_f64(X, ldx, W, w_type, ldw, C, ldc, Y, ldy, M, N, K, mech, sensitivity, epsilon,
                                    seed, stream_id, row0, workspace, workspace_bytes, stream=None):
    _check("splitee_masked_linear_fused_f64", load().splitee_masked_linear_fused_f64(
        _ptr(X), ldx, _ptr(W), w_type, ldw, _ptr(C), ldc, _ptr(Y), ldy, M, N, K, mech, sensitivity, epsilon, seed,
        stream_id, row0, _ptr(workspace), workspace_bytes, _stream(stream)))


def splitee_correction_f64(C, ldc, W, w_type, ldw, M, N, K, mech, sensitivity, epsilon, seed, stream_id, row0,
                           workspace, workspace_bytes, stream=None):
    _check("splitee_correction_f64", load().splitee_correction_f64(
        _ptr(C), ldc, _ptr(W), w_type, ldw, M, N, K, mech, sensitivity, epsilon, seed, stream_id, row0,
        _ptr(workspace), workspace_bytes, _stream(stream)))


def splitee_bank_path(directory, K, N, stream_id):
    buf = ctypes.create_string_buffer(4096)
    _check("splitee_bank_path", load().splitee_bank_path(os.fsencode(directory), K, N, stream_id, buf, 4096))
    return os.fsdecode(buf.value)


def splitee_bank_workspace_bytes(K, N, prec):
    return load().splitee_bank_workspace_bytes(K, N, prec)


def splitee_bank_create(path, W, w_type, ldw, K, N, mech, sensitivity, epsilon, seed, stream_id, row0, rows, prec,
                        workspace, workspace_bytes, stream=None):
    _check("splitee_bank_create", load().splitee_bank_create(
        os.fsencode(path), _ptr(W), w_type, ldw, K, N, mech, sensitivity, epsilon, seed, stream_id, row0, rows,
        prec, _ptr(workspace), workspace_bytes, _stream(stream)))


def splitee_bank_open(path):
    """Returns the bank handle (an integer address)."""
    h = ctypes.c_void_p()
    _check("splitee_bank_open", load().splitee_bank_open(os.fsencode(path), ctypes.byref(h)))
    return h.value


def splitee_bank_info(bank):
    info = BankInfo()
    _check("splitee_bank_info", load().splitee_bank_info(bank, ctypes.byref(info)))
    return info.as_dict()


def splitee_bank_load(bank, rows, C, ldc, dst_device, stream=None):
    """C: a device tensor (dst_device true) or a host address / contiguous CPU tensor;
    returns the first stream row of the loaded rows."""
    row0 = ctypes.c_int64()
    if dst_device:
        ptr = _ptr(C)
    else:
        ptr = C if isinstance(C, int) or C is None else C.data_ptr()
    _check("splitee_bank_load", load().splitee_bank_load(bank, rows, ptr, ldc, 1 if dst_device else 0,
                                                         ctypes.byref(row0), _stream(stream) if dst_device else None))
    return row0.value


def splitee_bank_close(bank):
    _check("splitee_bank_close", load().splitee_bank_close(bank))


def splitee_epilogue_workspace_bytes(M, N, K, prec, gated):
    return load().splitee_epilogue_workspace_bytes(M, N, K, prec, 1 if gated else 0)


def splitee_linear_epilogue(A, in_prec, lda, W, w_type, ldw, ep, Y, ldy, M, N, K, workspace, workspace_bytes,
                            stream=None):
    """ep: an Epilogue."""
    _check("splitee_linear_epilogue", load().splitee_linear_epilogue(
        _ptr(A), in_prec, lda, _ptr(W), w_type, ldw, ctypes.byref(ep), _ptr(Y), ldy, M, N, K, _ptr(workspace),
        workspace_bytes, _stream(stream)))


def splitee_grouped_linear(A, in_prec, lda, a_rows, row_index, offsets, experts, W, w_type, ldw, w_stride, ep, Y, ldy,
                           rows, N, K, stream=None):
    """ep: an Epilogue."""
    _check("splitee_grouped_linear", load().splitee_grouped_linear(
        _ptr(A), in_prec, lda, a_rows, _ptr(row_index), _ptr(offsets), experts, _ptr(W), w_type, ldw, w_stride,
        ctypes.byref(ep), _ptr(Y), ldy, rows, N, K, _stream(stream)))


def splitee_linear_plan_probe(rows, groups, dense, N, K, prec, gated):
    """(kind, rows, weight blocks, waves, splits, halved); see splitee_probe.h."""
    plan = (ctypes.c_int * 6)()
    _check("splitee_linear_plan_probe", load().splitee_linear_plan_probe(
        rows, groups, 1 if dense else 0, N, K, prec, 1 if gated else 0, ctypes.cast(plan, ctypes.c_void_p)))
    return tuple(plan)


def splitee_route_workspace_bytes(T, E, k):
    return load().splitee_route_workspace_bytes(T, E, k)


def splitee_route(logits, ldl, T, E, k, score, renorm, experts, weights, offsets, row_index, slot, workspace,
                  workspace_bytes, stream=None):
    _check("splitee_route", load().splitee_route(
        _ptr(logits), ldl, T, E, k, score, 1 if renorm else 0, _ptr(experts), _ptr(weights), _ptr(offsets),
        _ptr(row_index), _ptr(slot), _ptr(workspace), workspace_bytes, _stream(stream)))


def splitee_combine(H, h_type, ldh, h_rows, slot, weights, residual, ldres, Y, out_type, ldy, T, k, N, stream=None):
    _check("splitee_combine", load().splitee_combine(
        _ptr(H), h_type, ldh, h_rows, _ptr(slot), _ptr(weights), _ptr(residual), ldres, _ptr(Y), out_type, ldy, T, k,
        N, _stream(stream)))


# ------------------------------------------------- tensor-level conveniences

def _aligned_bytes(nbytes, device):
    buf = torch.empty(max(nbytes, 1) + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + max(nbytes, 1)]


def spectral_norm(W, iters, seed, stream_id, history=False, ws=None):
    """||W||_2 of a row-major N x K tensor by the power method (see splitee_spectral_norm)."""
    N, K = W.shape
    nbytes = splitee_spectral_norm_workspace_bytes(N, K, iters)
    if ws is None:
        ws = _aligned_bytes(nbytes, W.device)
    return splitee_spectral_norm(W, _wtype(W), W.stride(0), N, K, iters, seed, stream_id, ws, nbytes,
                                 history=history)


def workspace_f64(M, N, K, device="cuda"):
    """A 256-byte aligned workspace for the binary64 calls; returns (tensor, bytes)."""
    nbytes = splitee_f64_workspace_bytes(M, N, K)
    return _aligned_bytes(nbytes, device), nbytes


def correction_f64(W, M, mech, sensitivity, epsilon, seed, stream_id, row0=0, ws=None):
    N, K = W.shape
    C = torch.empty((M, N), dtype=torch.float64, device=W.device)
    if ws is None:
        ws = workspace_f64(M, N, K, W.device)
    splitee_correction_f64(C, N, W, _wtype(W), W.stride(0), M, N, K, mech, sensitivity, epsilon, seed, stream_id,
                           row0, ws[0], ws[1])
    return C


def masked_linear_fused_f64(X, W, C, mech, sensitivity, epsilon, seed, stream_id, row0=0, ws=None, Y=None):
    M, K = X.shape
    N = W.shape[0]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = workspace_f64(M, N, K, X.device)
    splitee_masked_linear_fused_f64(X, X.stride(0), W, _wtype(W), W.stride(0), C, C.stride(0), Y, Y.stride(0), M,
                                    N, K, mech, sensitivity, epsilon, seed, stream_id, row0, ws[0], ws[1])
    return Y


def bank_create(path, W, K, mech, sensitivity, epsilon, seed, stream_id, row0, rows, prec=SPLITEE_PREC_BF16X3):
    """Precompute and store the corrections of W (N x K) for `rows` stream rows."""
    N = W.shape[0]
    nbytes = splitee_bank_workspace_bytes(K, N, prec)
    ws = torch.zeros(nbytes + 256, dtype=torch.uint8, device=W.device)
    ws = ws[(-ws.data_ptr()) % 256:][:nbytes]
    splitee_bank_create(path, W, _wtype(W), W.stride(0), K, N, mech, sensitivity, epsilon, seed, stream_id, row0,
                        rows, prec, ws, nbytes)


def sensitivity(bound, alpha, beta=None, w_norm_a=0.0, w_norm_b=0.0):
    """Delta f of Theorem 1 (LN), 2 (ATT) or 3 (ACT) for float32 device vectors."""
    nbytes = splitee_sensitivity_workspace_bytes()
    ws = _aligned_bytes(nbytes, alpha.device)
    return splitee_sensitivity(bound, alpha.numel(), alpha, beta, w_norm_a, w_norm_b, ws, nbytes)


def workspace(M, N, K, prec, device="cuda", gemm_only=False):
    """A zeroed, 256-byte aligned workspace for the fused call / correction (or, with
    gemm_only, for splitee_masked_linear_unmask); returns (tensor, bytes)."""
    nbytes = (splitee_gemm_workspace_bytes if gemm_only else splitee_fused_workspace_bytes)(M, N, K, prec)
    ws = torch.zeros(max(nbytes, 1) + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + max(nbytes, 1)], nbytes


def tile_weights(W):
    """W (N x K bfloat16, row-major) in the tiled order, as TiledWeights."""
    _expect(W.dtype == torch.bfloat16, "W: expected bfloat16")
    N, K = W.shape
    data = torch.empty(splitee_tiled_weights_bytes(N, K) // 2, dtype=torch.bfloat16, device=W.device)
    splitee_tile_weights(W, W.stride(0), N, K, data)
    return TiledWeights(data, N, K)


def noise(M, K, mech, sensitivity, epsilon, seed, stream_id, row0=0, device="cuda"):
    eta = torch.empty((M, K), dtype=torch.float32, device=device)
    splitee_noise_gen(eta, K, M, K, mech, sensitivity, epsilon, seed, stream_id, row0)
    return eta


def mask(X, eta, prec):
    M, K = X.shape
    planes = 3 if prec == SPLITEE_PREC_BF16X3 else 1
    dt = torch.float32 if prec == SPLITEE_PREC_F32 else torch.int16
    Xt = torch.empty((planes, M, K), dtype=dt, device=X.device)
    splitee_mask(X, X.stride(0), eta, eta.stride(0), Xt, prec, K, M, K)
    return Xt


def masked_linear(Xt, prec, W):
    M, K = Xt.shape[-2:]
    N = W.shape[0]
    R = torch.empty((M, N), dtype=torch.float32, device=W.device)
    splitee_masked_linear(Xt, prec, K, W, _wtype(W), W.stride(0), R, N, M, N, K)
    return R


def noise_mask(X, prec, mech, sensitivity, epsilon, seed, stream_id, row0=0):
    M, K = X.shape
    planes = 3 if prec == SPLITEE_PREC_BF16X3 else 1
    dt = {SPLITEE_PREC_F32: torch.float32, SPLITEE_PREC_F64: torch.float64}.get(prec, torch.int16)
    Xt = torch.empty((planes, M, K), dtype=dt, device=X.device)
    splitee_noise_mask(X, X.stride(0), Xt, prec, K, M, K, mech, sensitivity, epsilon, seed,
                       stream_id, row0)
    return Xt


def masked_linear_unmask(Xt, prec, W, C, ws=None, Y=None):
    M, K = Xt.shape[-2:]
    N = W.shape[0]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float32, device=W.device)
    if ws is None:
        ws = workspace(M, N, K, prec, W.device, gemm_only=True)
    splitee_masked_linear_unmask(Xt, prec, K, W, _wtype(W), W.stride(0), C,
                                 C.stride(0) if C is not None else 0, Y, Y.stride(0), M, N, K,
                                 ws[0], ws[1])
    return Y


def unmask(R, C):
    M, N = R.shape
    Y = torch.empty((M, N), dtype=torch.float32, device=R.device)
    splitee_unmask(R, R.stride(0), C, C.stride(0), Y, N, M, N)
    return Y


def correction(W, M, mech, sensitivity, epsilon, seed, stream_id, row0=0, prec=SPLITEE_PREC_BF16X3,
               ws=None):
    N, K = W.shape
    C = torch.empty((M, N), dtype=torch.float32, device=W.device)
    if ws is None:
        ws = workspace(M, N, K, prec, W.device)
    splitee_correction(C, N, W, _wtype(W), W.stride(0), M, N, K, mech, sensitivity, epsilon, seed,
                       stream_id, row0, prec, ws[0], ws[1])
    return C


def masked_linear_fused(X, W, C, mech, sensitivity, epsilon, seed, stream_id, row0=0,
                        prec=SPLITEE_PREC_BF16X3, eta_override=None, ws=None, Y=None):
    M, K = X.shape
    N = W.shape[0]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = workspace(M, N, K, prec, X.device)
    splitee_masked_linear_fused(X, X.stride(0), W, _wtype(W), W.stride(0), C, C.stride(0), Y,
                                Y.stride(0), M, N, K, mech, sensitivity, epsilon, seed, stream_id,
                                row0, eta_override, prec, ws[0], ws[1])
    return Y


# ---------------------------------------- projections with an epilogue, and experts

_OUT = {torch.float32: SPLITEE_F32, torch.bfloat16: SPLITEE_BF16}


def _expect(ok, what):
    if not ok:
        raise ValueError(what)


def _here(*tensors):
    """The current device, whose stream the call takes: every tensor is on it."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("a tensor on device %d, the current device is %d" % (t.get_device(), dev))
    return dev


def _matrix(name, t, shape, dtype):
    """Leading dimension of a matrix of this shape and type."""
    s0, s1 = t.stride() if t.dim() == 2 else (0, 0)
    if t.shape != shape or t.dtype != dtype or (s1 != 1 and shape[1] > 1):
        raise ValueError("%s: expected %s of %s, columns contiguous" % (name, dtype, tuple(shape)))
    if shape[0] > 1:
        return s0
    per = 16 // dtype.itemsize
    return -(-shape[1] // per) * per  # of a single row no pitch is used


def _rows_out(rows, N, dtype, device):
    """(rows x N whose rows begin at multiples of 16 bytes, leading dimension)"""
    per = 16 // dtype.itemsize
    ld = -(-N // per) * per
    out = torch.empty((rows, ld), dtype=dtype, device=device)
    return (out if ld == N else out[:, :N]), ld


def _scratch(nbytes, device):
    """(address, tensor that holds it) of a 256-byte aligned workspace whose contents do not matter."""
    if not nbytes:
        return None, None
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if buf.data_ptr() % 256:
        buf = _aligned_bytes(nbytes, device)
    return buf.data_ptr(), buf


def _operand(A, prec):
    """(rows, K, leading dimension) of planes x rows x K as mask() returns them, or rows x K."""
    planes = 3 if prec == SPLITEE_PREC_BF16X3 else 1
    size = 4 if prec == SPLITEE_PREC_F32 else 2
    _expect(prec in (SPLITEE_PREC_F32, SPLITEE_PREC_BF16, SPLITEE_PREC_BF16X3), "A: precision F32, BF16 or BF16X3")
    _expect(A.dtype in ((torch.float32,) if size == 4 else (torch.bfloat16, torch.int16)), "A: dtype does not fit its precision")
    _expect(A.dim() == 3 and A.shape[0] == planes or A.dim() == 2 and planes == 1, "A: expected planes x rows x K")
    rows, K = A.shape[-2:]
    lda = K if not rows or not K else A.stride(-2) if rows > 1 else A.stride(0) if planes > 1 else K
    _expect(A.stride(-1) == 1 or K <= 1, "A: columns are not contiguous")
    _expect(planes == 1 or not A.numel() or A.stride(0) == rows * lda, "A: planes are not one after another")
    return rows, K, lda


def _epilogue(rows, N, NW, C, bias, act, gated, residual, out_dtype, bias_stride=0):
    _expect(out_dtype in _OUT, "out_dtype: float32 or bfloat16")
    ep = Epilogue(act=ACTS[act] if isinstance(act, str) else act, gated=1 if gated else 0, out_type=_OUT[out_dtype])
    if C is not None:
        ep.ldc = _matrix("C", C, (rows, NW), torch.float32)
        ep.C = C.data_ptr()
    if bias is not None:
        ep.bias, ep.bias_stride = bias.data_ptr(), bias_stride
    if residual is not None:
        ep.ldres = _matrix("residual", residual, (rows, N), out_dtype)
        ep.residual = residual.data_ptr()
    return ep


def _tiled_elements(N, K):
    return -(-N // 32) * -(-K // 64) * 2048


def _out_width(NW, gated):
    _expect(not gated or NW % 2 == 0, "W: a gated projection has as many gate as up rows")
    return NW // 2 if gated else NW


def linear_epilogue(A, prec, W, C=None, bias=None, act="none", gated=False, residual=None,
                    out_dtype=torch.float32, ws=None, Y=None):
    """epilogue(A W^T) (see splitee_linear_epilogue).  A: planes x M x K as mask() and noise_mask() return it, or
    M x K bfloat16 or float32; W: N (gated: 2 N) x K, a tensor or TiledWeights; act a name of ACTS."""
    M, K, lda = _operand(A, prec)
    NW = W.shape[0]
    _expect(len(W.shape) == 2 and W.shape[1] == K, "W: expected N x %d" % K)
    _expect(W.stride(1) == 1 or K <= 1, "W: columns are not contiguous")
    N, w_type = _out_width(NW, gated), _wtype(W)
    if w_type == SPLITEE_BF16_TILED:
        _expect(not M or W.data.is_contiguous() and W.data.numel() * W.data.element_size() >= 2 * _tiled_elements(NW, K),
                "W: less in one piece than its tiled order has")
    dev = _here(A, W.data if isinstance(W, TiledWeights) else W, C, bias, residual, Y)
    if bias is not None:
        _expect(tuple(bias.shape) == (NW,) and bias.dtype == torch.float32 and (NW < 2 or bias.stride(0) == 1),
                "bias: expected %d contiguous float32" % NW)
    ep = _epilogue(M, N, NW, C, bias, act, gated, residual, out_dtype)
    if Y is None:
        Y, ldy = _rows_out(M, N, out_dtype, A.device)
    else:
        ldy = _matrix("Y", Y, (M, N), out_dtype)
    lib = load()
    if ws is None:
        nbytes = lib.splitee_epilogue_workspace_bytes(M, N, K, prec, ep.gated)
        ws, held = _scratch(nbytes, A.device)
    else:
        ws, nbytes = _ptr(ws[0]), ws[1]
    _check("splitee_linear_epilogue", lib.splitee_linear_epilogue(
        A.data_ptr(), prec, lda, W.data_ptr(), w_type, W.stride(0) if NW > 1 and K else K, ctypes.byref(ep), Y.data_ptr(), ldy,
        M, N, K, ws, nbytes, torch._C._cuda_getCurrentRawStream(dev)))
    return Y


def grouped_linear(A, prec, W, offsets, row_index=None, C=None, bias=None, act="none", gated=False, residual=None,
                   out_dtype=torch.float32, Y=None):
    """Each expert's rows times its own W, with the epilogue (see splitee_grouped_linear).  W: experts x N (gated:
    2 N) x K, or the TiledWeights of tile_experts; offsets and row_index as route() returns them (without
    row_index, A is already in their order); bias experts x N (2 N)."""
    a_rows, K, lda = _operand(A, prec)
    tiled = isinstance(W, TiledWeights)
    _expect(len(W.shape) == (2 if tiled else 3) and W.shape[-1] == K, "W: expected experts x N x %d" % K)
    experts = (W.data if tiled else W).shape[0]
    NW = W.shape[-2]
    N, w_type = _out_width(NW, gated), _wtype(W)
    if tiled:
        _expect(W.data.dim() == 2 and W.data.element_size() == 2 and W.data.shape[1] >= _tiled_elements(NW, K)
                and W.data.stride(1) == 1, "W: expected experts x bfloat16 elements of tiled weights")
    dev = _here(A, W.data if tiled else W, offsets, row_index, C, bias, residual, Y)
    for name, t, n in (("offsets", offsets, experts + 1), ("row_index", row_index, None)):
        _expect(t is None or t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous() and n in (None, t.numel()),
                "%s: expected contiguous int32%s" % (name, " of experts + 1" if n else ""))
    rows = a_rows if row_index is None else row_index.numel()
    if tiled:
        ldw, w_stride = K, W.data.stride(0)
    else:
        _expect(W.stride(2) == 1 or K <= 1, "W: columns are not contiguous")
        ldw, w_stride = W.stride(1) if NW > 1 and K else K, W.stride(0) if experts > 1 and K else 0
    if bias is not None:
        _expect(tuple(bias.shape) == (experts, NW) and bias.dtype == torch.float32 and (NW < 2 or bias.stride(1) == 1),
                "bias: expected float32 of experts x %d" % NW)
    ep = _epilogue(rows, N, NW, C, bias, act, gated, residual, out_dtype, 0 if bias is None else bias.stride(0))
    if Y is None:
        Y, ldy = _rows_out(rows, N, out_dtype, A.device)
    else:
        ldy = _matrix("Y", Y, (rows, N), out_dtype)
    _check("splitee_grouped_linear", load().splitee_grouped_linear(
        A.data_ptr(), prec, lda, a_rows, None if row_index is None else row_index.data_ptr(), offsets.data_ptr(), experts,
        W.data_ptr(), w_type, ldw, w_stride, ctypes.byref(ep), Y.data_ptr(), ldy, rows, N, K,
        torch._C._cuda_getCurrentRawStream(dev)))
    return Y


def tile_experts(W):
    """experts x N x K bfloat16 in the tiled order, an expert a row of the TiledWeights' data."""
    _expect(W.dim() == 3 and W.dtype == torch.bfloat16 and (W.stride(2) == 1 or W.shape[2] <= 1),
            "W: expected bfloat16 of experts x N x K, columns contiguous")
    _here(W)
    E, N, K = W.shape
    data = torch.empty((E, splitee_tiled_weights_bytes(N, K) // 2), dtype=torch.bfloat16, device=W.device)
    for e in range(E):
        splitee_tile_weights(W[e], W.stride(1) if N > 1 else K, N, K, data[e])
    return TiledWeights(data, N, K)


class Routes(typing.NamedTuple):
    """What splitee_route writes."""
    experts: torch.Tensor    # T x k int32
    weights: torch.Tensor    # T x k float32
    offsets: torch.Tensor    # experts + 1 int32
    row_index: torch.Tensor  # T * k int32
    slot: torch.Tensor       # T x k int32


def route(logits, k, score="softmax", renorm=True, ws=None):
    """The k experts of every token and the order of the rows (see splitee_route).  logits: T x experts float32."""
    _expect(logits.dim() == 2 and logits.dtype == torch.float32, "logits: expected float32 of tokens x experts")
    T, E = logits.shape
    _expect(logits.stride(1) == 1 or E <= 1, "logits: columns are not contiguous")
    here = _here(logits)
    dev, i32 = logits.device, torch.int32
    r = Routes(torch.empty((T, k), dtype=i32, device=dev), torch.empty((T, k), dtype=torch.float32, device=dev),
               torch.empty(E + 1, dtype=i32, device=dev), torch.empty(T * k, dtype=i32, device=dev),
               torch.empty((T, k), dtype=i32, device=dev))
    lib = load()
    if ws is None:
        nbytes = lib.splitee_route_workspace_bytes(T, E, k)
        ws, held = _scratch(nbytes, dev)
    else:
        ws, nbytes = _ptr(ws[0]), ws[1]
    _check("splitee_route", lib.splitee_route(
        logits.data_ptr(), logits.stride(0) if T > 1 else E, T, E, k, SCORES[score] if isinstance(score, str) else score,
        1 if renorm else 0, r.experts.data_ptr(), r.weights.data_ptr(), r.offsets.data_ptr(), r.row_index.data_ptr(),
        r.slot.data_ptr(), ws, nbytes, torch._C._cuda_getCurrentRawStream(here)))
    return r


def combine(H, slot, weights, residual=None, out_dtype=torch.float32, Y=None):
    """Y[t] = residual[t] + sum_j weights[t, j] H[slot[t, j]] (see splitee_combine)."""
    _expect(H.dim() == 2 and H.dtype in _OUT and out_dtype in _OUT, "H, out_dtype: float32 or bfloat16")
    _expect(slot.dim() == 2 and slot.dtype == torch.int32 and slot.is_contiguous() and weights.shape == slot.shape
            and weights.dtype == torch.float32 and weights.is_contiguous(),
            "slot, weights: expected contiguous int32 and float32 of tokens x k")
    (h_rows, N), (T, k) = H.shape, slot.shape
    dev = _here(H, slot, weights, residual, Y)
    ldh = _matrix("H", H, (h_rows, N), H.dtype)
    ldres = _matrix("residual", residual, (T, N), out_dtype) if residual is not None else 0
    if Y is None:
        Y, ldy = _rows_out(T, N, out_dtype, H.device)
    else:
        ldy = _matrix("Y", Y, (T, N), out_dtype)
    _check("splitee_combine", load().splitee_combine(
        H.data_ptr(), _OUT[H.dtype], ldh, h_rows, slot.data_ptr(), weights.data_ptr(),
        None if residual is None else residual.data_ptr(), ldres, Y.data_ptr(), _OUT[out_dtype], ldy, T, k, N,
        torch._C._cuda_getCurrentRawStream(dev)))
    return Y


def _mask_planes(X, rows, K, prec, mech, sensitivity, epsilon, seed, stream_id, row0, device):
    """noise_mask of X, or (X None) of zeros: the planes of the mask itself."""
    planes = 3 if prec == SPLITEE_PREC_BF16X3 else 1
    Xt = torch.empty((planes, rows, K), dtype=torch.float32 if prec == SPLITEE_PREC_F32 else torch.int16, device=device)
    splitee_noise_mask(X, K if X is None or rows < 2 else X.stride(0), Xt, prec, K, rows, K, mech, sensitivity, epsilon, seed,
                       stream_id, row0)
    return Xt


def expert_ffn(X, logits, k, W_gate_up, W_down, mech=SPLITEE_MECH_NONE, sensitivity=0.0, epsilon=1.0, seed=0, stream_id=0,
               row0=0, prec=SPLITEE_PREC_BF16X3, act="silu", score="softmax", renorm=True, residual=None,
               out_dtype=torch.float32):
    """The feed-forward part of a mixture-of-experts layer under masks: route the tokens, mask them, the experts' gate
    and up projections unmasked and gated, mask the result, the experts' down projections unmasked, and the
    weighted sum, plus the residual.

    X: tokens x K float32; logits: tokens x experts float32; W_gate_up: experts x 2 N x K and W_down: experts x D x N,
    bfloat16 tensors or the TiledWeights of tile_experts (float32 with SPLITEE_PREC_F32), K and N multiples of 8.  The
    masks are rows row0 .. of noise stream stream_id (gate and up: a token has one mask for all its experts) and rows
    row0 k .. of stream stream_id + 1 (down: one for each row in the router's order).  As in the fused call the
    corrections are formed on this GPU, here once the rows' experts are known; SPLITEE_MECH_NONE is the split without
    noise, which has none."""
    _expect(X.dim() == 2 and X.dtype == torch.float32 and (X.stride(1) == 1 or X.shape[1] <= 1),
            "X: expected float32 of tokens x K, columns contiguous")
    T, K = X.shape
    D, N = W_down.shape[-2:]
    _expect(logits.dim() == 2 and logits.shape[0] == T, "logits: expected %d tokens x experts" % T)
    _expect(tuple(W_gate_up.shape[-2:]) == (2 * N, K), "W_gate_up: expected experts x %d x %d" % (2 * N, K))
    _wtype(W_gate_up, "W_gate_up")
    _wtype(W_down, "W_down")
    if residual is not None:
        _matrix("residual", residual, (T, D), out_dtype)
    _here(X, logits, residual, *(W.data if isinstance(W, TiledWeights) else W for W in (W_gate_up, W_down)))
    r = route(logits, k, score=score, renorm=renorm)
    noise_args = (mech, sensitivity, epsilon, seed)
    masked = mech != SPLITEE_MECH_NONE
    exact = SPLITEE_PREC_F32 if prec == SPLITEE_PREC_F32 else SPLITEE_PREC_BF16X3  # of a correction

    def projection(A, rows, width, W, sid, first, index, **epilogue):
        C = None
        if masked:
            eta = _mask_planes(None, rows, width, exact, *noise_args, sid, first, X.device)
            C = grouped_linear(eta, exact, W, r.offsets, row_index=index)
        At = _mask_planes(A, rows, width, prec, *noise_args, sid, first, X.device)
        return grouped_linear(At, prec, W, r.offsets, row_index=index, C=C, **epilogue)

    H = projection(X, T, K, W_gate_up, stream_id, row0, r.row_index, act=act, gated=True)
    R = projection(H, T * k, N, W_down, stream_id + 1, row0 * k, None)
    return combine(R, r.slot, r.weights, residual=residual, out_dtype=out_dtype)
