"""ctypes binding of libgls.so (C ABI in include/gls.h).  Argument marshalling only."""
import ctypes as C
import importlib.util
import math
import os
import shutil
import subprocess
import sysconfig
import threading
import warnings
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
_SRC_DIR = os.path.join(_HERE, "csrc")
_LIB = os.path.join(_HERE, "libgls.so")
# The compiled calls use the layout of this Python's and this torch's objects: a module made for others has
# another name and is not loaded.
_CALLS_LIB = os.path.join(_HERE, "gls_torch_calls.%s-torch%s-cuda%s.so" % (
    sysconfig.get_config_var("SOABI"), torch.__version__, torch.version.cuda))

COMBINE_ACTIVE, COMBINE_ALL, NO_BONUS = 0, 1, 2
VERIFY_ALL_ROWS, VERIFY_ACTIVE_ROWS = 4, 8  # how the dense verify call walks Algorithm 2
VERIFY_FIRST_PHASE, VERIFY_REST = 16, 32   # the walk in phases as two calls (rows fetched on demand)
VERIFY_THREE_PHASES = 64                   # positions 1 and 2 as a phase of their own
NOISE_SHARED_ACROSS_K = 1
DEV_EMPTY_SUPPORT, DEV_BAD_TOKEN, DEV_BAD_SETTING = 1, 2, 4
EMBED_ACCUMULATE = 1
MAX_GIVEN = 64  # tokens per row of token_logprobs
F32, BF16 = 0, 1

_lock = threading.Lock()
_lib = None
_calls = None


class GlsError(RuntimeError):
    pass


def lib_path():
    return _LIB


def _sources():
    return sorted(os.path.join(_SRC_DIR, f) for f in os.listdir(_SRC_DIR)
                  if f.endswith((".cu", ".cuh"))) + [os.path.join(_ROOT, "include", "gls.h")]


def _build_calls(force):
    """Compile csrc/torch_calls.cpp, a Python module over torch's headers, with the host compiler."""
    srcs = [os.path.join(_SRC_DIR, "torch_calls.cpp"), os.path.join(_ROOT, "include", "gls.h")]
    if (not force and os.path.exists(_CALLS_LIB)
            and os.path.getmtime(_CALLS_LIB) >= max(os.path.getmtime(s) for s in srcs)):
        return
    at = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")))
    tmp = _CALLS_LIB + ".tmp%d" % os.getpid()
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                    "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
                    "-I" + os.path.join(at, "include"),
                    "-I" + os.path.join(at, "include", "torch", "csrc", "api", "include"),
                    "-I" + os.path.join(cuda, "include"), "-I" + sysconfig.get_paths()["include"], "-o", tmp, srcs[0],
                    "-L" + os.path.join(at, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch",
                    "-ltorch_python"], check=True)
    os.replace(tmp, _CALLS_LIB)


def build(force=False, verbose=False, debug_bounds=False):
    """Compile csrc/*.cu into libgls.so for sm_100a with nvcc (cross-compiles without a GPU), and
    csrc/torch_calls.cpp beside it; warns when the latter can not be compiled (see _GeneralWay)."""
    srcs = _sources()
    if force or not os.path.exists(_LIB) or os.path.getmtime(_LIB) < max(os.path.getmtime(s) for s in srcs):
        cus = [s for s in srcs if s.endswith(".cu")]
        tmp = _LIB + ".tmp%d" % os.getpid()
        cmd = ["nvcc", "--threads", "4", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
               "-shared", "-Xcompiler", "-fPIC", "-o", tmp] + cus
        if debug_bounds or os.environ.get("GLS_DEBUG_BOUNDS") == "1":
            cmd.insert(1, "-DGLS_DEBUG_BOUNDS")  # range checks of the kernels' own indices
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        subprocess.run(cmd, check=True)
        os.replace(tmp, _LIB)
    try:
        _build_calls(force)
    except (OSError, subprocess.CalledProcessError) as e:
        _without_calls(e)
    return _LIB


class _GeneralWay:
    """Stands in for the compiled calls where they can not be had: declines every call, which binding.py
    then makes through ctypes, with the same kernels and results and 10 us more of host time."""

    def __getattr__(self, name):
        return self._decline

    @staticmethod
    def _decline(*args):
        return None


def _without_calls(error):
    warnings.warn("%s can not be used (%s): the calls that it shortens are made through ctypes"
                  % (os.path.basename(_CALLS_LIB), error), RuntimeWarning, stacklevel=3)


def _load_calls(L):
    """The compiled calls with the entry points of the library L."""
    try:
        if not os.path.exists(_CALLS_LIB):
            _build_calls(False)
        spec = importlib.util.spec_from_file_location("gls_torch_calls", _CALLS_LIB)
        calls = importlib.util.module_from_spec(spec)
        calls.entry_points(*(C.cast(getattr(L, "gls_" + n), C.c_void_p).value for n in (
            "token_logprobs", "emitted_logprobs", "token_logprobs_backward", "embed_tokens",
            "embed_tokens_backward_workspace_bytes", "embed_tokens_backward", "sample_tokens", "head_logits",
            "head_logits_workspace_bytes", "embed_tokens_int4")))
        return calls
    except (ImportError, OSError, TypeError, subprocess.CalledProcessError) as e:  # TypeError: made from older sources
        _without_calls(e)
        return _GeneralWay()


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("stride_b", C.c_int64),
                ("stride_k", C.c_int64), ("stride_j", C.c_int64)]


class _SparseRows(C.Structure):
    _fields_ = [("token_ids", C.c_void_p), ("logits", C.c_void_p), ("stride_b", C.c_int64),
                ("stride_k", C.c_int64), ("stride_j", C.c_int64), ("M", C.c_int32)]


class _Sampling(C.Structure):
    _fields_ = [("inv_temp", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float),
                ("inv_temp_rows", C.c_void_p), ("top_k_rows", C.c_void_p), ("top_p_rows", C.c_void_p),
                ("min_p_rows", C.c_void_p), ("inv_temp_stride", C.c_int64 * 3), ("top_k_stride", C.c_int64 * 3),
                ("top_p_stride", C.c_int64 * 3), ("min_p_stride", C.c_int64 * 3)]


class _Int4(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("code_stride", C.c_int64), ("scales", C.c_void_p),
                ("scale_dtype", C.c_int32), ("scale_stride", C.c_int64), ("zeros", C.c_void_p),
                ("zero_stride", C.c_int64), ("V", C.c_int64), ("D", C.c_int64), ("group", C.c_int32)]


class _Noise(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("seq_base", C.c_uint32), ("seq_ids", C.c_void_p),
                ("pos_base", C.c_uint32), ("noise_spec", C.c_uint32), ("rounds", C.c_uint32),
                ("flags", C.c_uint32)]


def load():
    """Load libgls.so (building it if it is not there), and the compiled calls beside it where they can be had."""
    global _lib, _calls
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(_LIB):
            build()
        L = C.CDLL(_LIB)
        L.gls_version.restype = C.c_int
        L.gls_status_string.restype = C.c_char_p
        L.gls_status_string.argtypes = [C.c_int]
        L.gls_workspace_bytes.restype = C.c_size_t
        L.gls_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int64]
        L.gls_draft_sample.restype = C.c_int
        L.gls_draft_sample.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p,
            C.c_void_p]
        L.gls_static_scratch_bytes.restype = C.c_size_t
        L.gls_draft_sample_static.restype = C.c_int
        L.gls_draft_sample_static.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.gls_draft_sample_sparse.restype = C.c_int
        L.gls_draft_sample_sparse.argtypes = [
            C.POINTER(_SparseRows), C.c_int, C.c_int, C.c_int, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.gls_target_sample_verify_sparse.restype = C.c_int
        L.gls_target_sample_verify_sparse.argtypes = [
            C.POINTER(_SparseRows), C.c_int, C.c_int, C.c_int, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p]
        L.gls_target_sample_verify.restype = C.c_int
        L.gls_target_sample_verify.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.gls_draft_verify_workspace_bytes.restype = C.c_size_t
        L.gls_draft_verify_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64]
        L.gls_draft_verify.restype = C.c_int
        L.gls_draft_verify.argtypes = [
            C.POINTER(_Rows), C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float,
            C.c_void_p, C.c_float, C.POINTER(_Noise), C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.gls_topm_workspace_bytes.restype = C.c_size_t
        L.gls_topm_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int]
        L.gls_draft_sample_topm.restype = C.c_int
        L.gls_draft_sample_topm.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p,
            C.c_void_p]
        L.gls_target_sample_verify_topm.restype = C.c_int
        L.gls_target_sample_verify_topm.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int, C.c_float, C.c_void_p,
            C.POINTER(_Noise), C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.gls_compress_gaussian_workspace_bytes.restype = C.c_size_t
        L.gls_compress_gaussian_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int64]
        L.gls_compress_gaussian.restype = C.c_int
        L.gls_compress_gaussian.argtypes = [
            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_int, C.c_int64,
            C.c_int, C.c_double, C.c_double, C.c_double, C.POINTER(_Noise), C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
            C.c_void_p, C.c_void_p]
        L.gls_compress_select.restype = C.c_int
        L.gls_compress_select.argtypes = [
            C.POINTER(_Rows), C.POINTER(_Rows), C.c_void_p, C.c_int64, C.c_int, C.c_int,
            C.c_int64, C.POINTER(_Noise), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.gls_token_logprobs.restype = C.c_int
        L.gls_token_logprobs.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p, C.c_void_p,
            C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p]
        L.gls_emitted_logprobs.restype = C.c_int
        L.gls_emitted_logprobs.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p, C.c_void_p,
            C.c_uint32, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p]
        L.gls_token_logprobs_backward.restype = C.c_int
        L.gls_token_logprobs_backward.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.c_float, C.c_void_p, C.c_void_p,
            C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p, C.POINTER(_Rows), C.c_void_p]
        L.gls_embed_tokens.restype = C.c_int
        L.gls_embed_tokens.argtypes = [
            C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_float,
            C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.gls_embed_tokens_backward_workspace_bytes.restype = C.c_size_t
        L.gls_embed_tokens_backward_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int64]
        L.gls_embed_tokens_backward.restype = C.c_int
        L.gls_embed_tokens_backward.argtypes = [
            C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_float,
            C.c_void_p, C.c_int, C.c_int64, C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.gls_sample_tokens.restype = C.c_int
        L.gls_sample_tokens.argtypes = [
            C.POINTER(_Rows), C.c_int, C.c_int, C.c_int, C.c_int64, C.POINTER(_Sampling), C.c_void_p, C.c_void_p,
            C.c_void_p, C.c_void_p, C.c_void_p]
        L.gls_quantize_table.restype = C.c_int
        L.gls_quantize_table.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.POINTER(_Int4), C.c_void_p]
        L.gls_head_logits.restype = C.c_int
        L.gls_head_logits.argtypes = [
            C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.POINTER(_Int4), C.c_void_p, C.c_int, C.c_int64, C.c_void_p,
            C.c_size_t, C.c_void_p]
        L.gls_head_logits_workspace_bytes.restype = C.c_size_t
        L.gls_head_logits_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int]
        L.gls_embed_tokens_int4.restype = C.c_int
        L.gls_embed_tokens_int4.argtypes = [
            C.POINTER(_Int4), C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_void_p]
        _calls = _load_calls(L)
        _lib = L
        return _lib


def debug_bounds():
    """(compiled in?, [count, first site, value, limit]) of the library's index self-check."""
    out = (C.c_uint32 * 4)()
    L = load()
    L.gls_debug_bounds.restype = C.c_int
    rc = int(L.gls_debug_bounds(out))
    return rc, [int(x) for x in out]


def version():
    return int(load().gls_version())


def status_string(rc):
    return load().gls_status_string(int(rc)).decode()


def workspace_bytes(B, K, J, V):
    return int(load().gls_workspace_bytes(int(B), int(K), int(J), int(V)))


def _check(rc):
    if rc != 0:
        raise GlsError(status_string(rc))


def _rows(t, lead):
    """gls_rows_t of a tensor whose last dim is contiguous; `lead` leading dims give strides."""
    if not t.is_cuda:
        raise GlsError("libgls takes device tensors; there is no CPU path")
    if t.dtype == torch.float32:
        dt = F32
    elif t.dtype == torch.bfloat16:
        dt = BF16
    else:
        raise GlsError("logits must be float32 or bfloat16")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise GlsError("the token dimension must be contiguous")
    st = [t.stride(d) for d in range(lead)] + [0] * (3 - lead)
    return _Rows(t.data_ptr(), dt, st[0], st[1], st[2])


def _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, flags):
    ptr = None
    if seq_ids is not None:
        if seq_ids.dtype != torch.int32 or not seq_ids.is_cuda or not seq_ids.is_contiguous():
            raise GlsError("seq_ids must be a contiguous int32 device tensor (bit pattern = uint32)")
        ptr = seq_ids.data_ptr()
    return _Noise(int(seed) & (2**64 - 1), int(seq_base), ptr, int(pos_base), int(spec),
                  int(rounds), int(flags))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _workspace(workspace, need, device):
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace


def _wrote(*given):
    """Counts what a call wrote into tensors that its caller gave as a change of them, as torch's own in-place
    operations do: a backward pass that saved one (the tokens of a lookup, say) then refuses it."""
    increment_version([t for t in given if t is not None])


def draft_sample(logits, inv_temp=1.0, inv_temp_per_draft=None, seed=0, seq_base=0, seq_ids=None,
                 pos_base=0, spec=4, rounds=10, noise_flags=0, want_scores=True, workspace=None,
                 status=None, out_tokens=None, out_scores=None):
    """logits [B,K,J,V] (device, fp32/bf16) -> (tokens int32 [B,K,J], scores fp32 [B,K,J] | None)."""
    L = load()
    B, K, J, V = logits.shape
    dev = logits.device
    rows = _rows(logits, 3)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    given = out_tokens, out_scores
    if out_tokens is None:
        out_tokens = torch.empty((B, K, J), dtype=torch.int32, device=dev)
    if out_scores is None and want_scores:
        out_scores = torch.empty((B, K, J), dtype=torch.float32, device=dev)
    need = workspace_bytes(B, K, J, V)
    workspace = _workspace(workspace, need, dev)
    itk = None
    if inv_temp_per_draft is not None:
        itk = (C.c_float * K)(*[float(x) for x in inv_temp_per_draft])
    _check(L.gls_draft_sample(C.byref(rows), B, K, J, V, float(inv_temp),
                              C.cast(itk, C.c_void_p) if itk is not None else None, C.byref(nz),
                              _ptr(out_tokens), _ptr(out_scores), workspace.data_ptr(),
                              workspace.numel(), _ptr(status), _stream()))
    _wrote(*given)
    return out_tokens, out_scores


def static_scratch_bytes():
    return int(load().gls_static_scratch_bytes())


def draft_sample_static(logits, out_tokens, out_scores=None, inv_temp=1.0, inv_temp_per_draft=None,
                        seed=0, seq_base=0, seq_ids=None, pos_base=0, spec=4, rounds=10,
                        noise_flags=0, status=None):
    """gls_draft_sample_static: draft_sample for callers that may not allocate device memory.

    The caller passes the outputs (int32 [B,K,J], optional fp32 [B,K,J]); this wrapper creates no
    tensor and the library uses its built-in scratch buffer.  Raises GlsError when the problem
    needs more scratch than static_scratch_bytes()."""
    L = load()
    B, K, J, V = logits.shape
    rows = _rows(logits, 3)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    itk = None
    if inv_temp_per_draft is not None:
        itk = (C.c_float * K)(*[float(x) for x in inv_temp_per_draft])
    _check(L.gls_draft_sample_static(C.byref(rows), B, K, J, V, float(inv_temp),
                                     C.cast(itk, C.c_void_p) if itk is not None else None,
                                     C.byref(nz), _ptr(out_tokens), _ptr(out_scores), _ptr(status),
                                     _stream()))
    _wrote(out_tokens, out_scores)
    return out_tokens, out_scores


def _sparse(ids, logits):
    """gls_sparse_rows_t of ids int32 [B,K,J,M] and logits fp32 with the same shape and strides."""
    if not (ids.is_cuda and logits.is_cuda):
        raise GlsError("libgls takes device tensors; there is no CPU path")
    if ids.dtype != torch.int32 or logits.dtype != torch.float32:
        raise GlsError("sparse rows are int32 token ids and float32 logits")
    if ids.shape != logits.shape or ids.stride() != logits.stride():
        raise GlsError("token_ids and logits must share shape and strides")
    if ids.stride(-1) != 1 and ids.shape[-1] > 1:
        raise GlsError("the kept-token dimension must be contiguous")
    return _SparseRows(ids.data_ptr(), logits.data_ptr(), ids.stride(0), ids.stride(1),
                       ids.stride(2), ids.shape[3])


def draft_sample_sparse(token_ids, logits, inv_temp=1.0, inv_temp_per_draft=None, seed=0,
                        seq_base=0, seq_ids=None, pos_base=0, spec=4, rounds=10, noise_flags=0,
                        want_scores=True, status=None):
    """Sparse rows (kept token ids and their logits, [B,K,J,M]) -> (vocabulary ids int32 [B,K,J],
    scores fp32 [B,K,J] | None).  Same races as draft_sample on the row masked to the kept tokens."""
    L = load()
    B, K, J, M = token_ids.shape
    rows = _sparse(token_ids, logits)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    dev = token_ids.device
    out_tokens = torch.empty((B, K, J), dtype=torch.int32, device=dev)
    out_scores = torch.empty((B, K, J), dtype=torch.float32, device=dev) if want_scores else None
    itk = None
    if inv_temp_per_draft is not None:
        itk = (C.c_float * K)(*[float(x) for x in inv_temp_per_draft])
    _check(L.gls_draft_sample_sparse(C.byref(rows), B, K, J, float(inv_temp),
                                     C.cast(itk, C.c_void_p) if itk is not None else None,
                                     C.byref(nz), _ptr(out_tokens), _ptr(out_scores), _ptr(status),
                                     _stream()))
    return out_tokens, out_scores


def target_sample_verify_sparse(token_ids, logits, draft_tokens, inv_temp=1.0, flags=0, seed=0,
                                seq_base=0, seq_ids=None, pos_base=0, spec=4, rounds=10,
                                noise_flags=0, want_scores=True, status=None):
    """Sparse target rows [B,K,J,M] (J = L+1, or L with NO_BONUS) and draft_tokens int32 [B,K,L]
    -> dict(tokens [B,J], tau [B], accept [B,K,L], scores [B,J] | None)."""
    L = load()
    B, K, J, M = token_ids.shape
    Ld = J if (flags & NO_BONUS) else J - 1
    rows = _sparse(token_ids, logits)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    dev = token_ids.device
    if Ld > 0:
        if draft_tokens.dtype != torch.int32 or not draft_tokens.is_contiguous():
            raise GlsError("draft_tokens must be contiguous int32")
        assert tuple(draft_tokens.shape) == (B, K, Ld)
    out = dict(tokens=torch.empty((B, J), dtype=torch.int32, device=dev),
               tau=torch.empty((B,), dtype=torch.int32, device=dev),
               accept=torch.empty((B, K, Ld), dtype=torch.uint8, device=dev),
               scores=torch.empty((B, J), dtype=torch.float32, device=dev) if want_scores else None)
    _check(L.gls_target_sample_verify_sparse(
        C.byref(rows), B, K, Ld, float(inv_temp), _ptr(draft_tokens) if Ld > 0 else None,
        C.byref(nz), int(flags), _ptr(out["tokens"]), _ptr(out["tau"]),
        _ptr(out["accept"]) if Ld > 0 else None, _ptr(out.get("scores")), _ptr(status), _stream()))
    return out


def topm_workspace_bytes(B, K, J, M):
    return int(load().gls_topm_workspace_bytes(int(B), int(K), int(J), int(M)))


def _topm_lists(workspace, B, K, J, M):
    """Views of the kept (ids int32, logits fp32) lists [B,K,J,M] a top-M call left in its workspace."""
    n = B * K * J * M
    off = (n * 4 + 255) // 256 * 256
    ids = workspace[:n * 4].view(torch.int32).view(B, K, J, M)
    lg = workspace[off:off + n * 4].view(torch.float32).view(B, K, J, M)
    return ids, lg


def draft_sample_topm(logits, M, inv_temp=1.0, inv_temp_per_draft=None, seed=0, seq_base=0,
                      seq_ids=None, pos_base=0, spec=4, rounds=10, noise_flags=0, want_scores=True,
                      workspace=None, status=None):
    """Dense logits [B,K,J,V] truncated to their M largest per row, then draft_sample_sparse.

    Returns (tokens int32 [B,K,J], scores | None, (kept ids, kept logits) views [B,K,J,M])."""
    L = load()
    B, K, J, V = logits.shape
    dev = logits.device
    rows = _rows(logits, 3)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    out_tokens = torch.empty((B, K, J), dtype=torch.int32, device=dev)
    out_scores = torch.empty((B, K, J), dtype=torch.float32, device=dev) if want_scores else None
    workspace = _workspace(workspace, topm_workspace_bytes(B, K, J, M), dev)
    itk = None
    if inv_temp_per_draft is not None:
        itk = (C.c_float * K)(*[float(x) for x in inv_temp_per_draft])
    _check(L.gls_draft_sample_topm(C.byref(rows), B, K, J, V, int(M), float(inv_temp),
                                   C.cast(itk, C.c_void_p) if itk is not None else None,
                                   C.byref(nz), _ptr(out_tokens), _ptr(out_scores),
                                   workspace.data_ptr(), workspace.numel(), _ptr(status), _stream()))
    _wrote(workspace)  # views of it were returned
    return out_tokens, out_scores, _topm_lists(workspace, B, K, J, M)


def target_sample_verify_topm(logits, draft_tokens, M, inv_temp=1.0, flags=0, seed=0, seq_base=0,
                              seq_ids=None, pos_base=0, spec=4, rounds=10, noise_flags=0,
                              want_scores=True, workspace=None, status=None):
    """Dense target logits [B,K,J,V] truncated to their M largest per row, then
    target_sample_verify_sparse.  Returns dict(tokens, tau, accept, scores | None)."""
    L = load()
    B, K, J, V = logits.shape
    Ld = J if (flags & NO_BONUS) else J - 1
    dev = logits.device
    rows = _rows(logits, 3)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    if Ld > 0:
        if draft_tokens.dtype != torch.int32 or not draft_tokens.is_contiguous():
            raise GlsError("draft_tokens must be contiguous int32")
        assert tuple(draft_tokens.shape) == (B, K, Ld)
    out = dict(tokens=torch.empty((B, J), dtype=torch.int32, device=dev),
               tau=torch.empty((B,), dtype=torch.int32, device=dev),
               accept=torch.empty((B, K, Ld), dtype=torch.uint8, device=dev),
               scores=torch.empty((B, J), dtype=torch.float32, device=dev) if want_scores else None)
    workspace = _workspace(workspace, topm_workspace_bytes(B, K, J, M), dev)
    _check(L.gls_target_sample_verify_topm(
        C.byref(rows), B, K, Ld, V, int(M), float(inv_temp),
        _ptr(draft_tokens) if Ld > 0 else None, C.byref(nz), int(flags), _ptr(out["tokens"]),
        _ptr(out["tau"]), _ptr(out["accept"]) if Ld > 0 else None, _ptr(out.get("scores")),
        workspace.data_ptr(), workspace.numel(), _ptr(status), _stream()))
    _wrote(workspace)
    return out


def target_sample_verify(logits, draft_tokens, inv_temp=1.0, flags=0, seed=0, seq_base=0,
                         seq_ids=None, pos_base=0, spec=4, rounds=10, noise_flags=0,
                         want_scores=True, workspace=None, status=None, out=None):
    """logits [B,K,J,V], draft_tokens int32 [B,K,L]; J = L+1 (L with NO_BONUS).

    Returns dict(tokens [B,J], tau [B], accept [B,K,L], scores [B,J] | None)."""
    L = load()
    B, K, J, V = logits.shape
    Ld = J if (flags & NO_BONUS) else J - 1
    dev = logits.device
    rows = _rows(logits, 3)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    if Ld > 0:
        if draft_tokens.dtype != torch.int32 or not draft_tokens.is_contiguous():
            raise GlsError("draft_tokens must be contiguous int32")
        assert tuple(draft_tokens.shape) == (B, K, Ld)
    given = out
    if out is None:
        out = dict(tokens=torch.empty((B, J), dtype=torch.int32, device=dev),
                   tau=torch.empty((B,), dtype=torch.int32, device=dev),
                   accept=torch.empty((B, K, Ld), dtype=torch.uint8, device=dev),
                   scores=torch.empty((B, J), dtype=torch.float32, device=dev)
                   if want_scores else None)
    need = workspace_bytes(B, K, J, V)
    workspace = _workspace(workspace, need, dev)
    _check(L.gls_target_sample_verify(
        C.byref(rows), B, K, Ld, V, float(inv_temp), _ptr(draft_tokens) if Ld > 0 else None,
        C.byref(nz), int(flags), _ptr(out["tokens"]), _ptr(out["tau"]),
        _ptr(out["accept"]) if Ld > 0 else None, _ptr(out.get("scores")), workspace.data_ptr(),
        workspace.numel(), _ptr(status), _stream()))
    if given is not None:
        _wrote(*given.values())
    return out


def copy_rows_to_device(dst, src, stream=None):
    """dst (device) and src (pinned host): tensors of the same shape [n, row] and dtype whose rows
    are contiguous and a constant stride apart (e.g. t[:, :, 0].flatten(0, 1) of a [B,K,J,V]
    tensor): one strided host-to-device copy on `stream` (default: the current stream)."""
    assert dst.dim() == 2 and dst.shape == src.shape and dst.dtype == src.dtype
    assert dst.is_cuda and not src.is_cuda
    if dst.shape[1] > 1 and (dst.stride(1) != 1 or src.stride(1) != 1):
        raise GlsError("rows must be contiguous")
    es = dst.element_size()
    lib = load()
    lib.gls_copy_rows_to_device.restype = C.c_int
    lib.gls_copy_rows_to_device.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_size_t,
                                            C.c_size_t, C.c_void_p]
    n, row = dst.shape
    st = stream.cuda_stream if stream is not None else _stream()
    _check(lib.gls_copy_rows_to_device(dst.data_ptr(), max(dst.stride(0), row) * es, src.data_ptr(),
                                       max(src.stride(0), row) * es, row * es, n, st))
    _wrote(dst)


def verify_walk(target_logits, L, flags=0, spec=4):
    """1 if target_sample_verify would walk Algorithm 2 in phases for these rows (reading the rows
    of active drafts only), 0 if it would race every row first; GlsError for refused arguments."""
    B, K, J, V = target_logits.shape
    lib = load()
    lib.gls_verify_walk.restype = C.c_int
    lib.gls_verify_walk.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int,
                                    C.c_uint32]
    rc = int(lib.gls_verify_walk(BF16 if target_logits.dtype == torch.bfloat16 else F32,
                                 int(target_logits.stride(1) != 0), B, K, int(L), V, int(spec), int(flags)))
    if rc < 0:
        raise GlsError("gls_verify_walk: arguments that the verify call refuses")
    return rc


def verify_phases(target_logits, L, flags=0, spec=4):
    """Phase boundaries of target_sample_verify's walk for these rows: [] if every row is raced,
    else [e0, e1, ...] with phase p covering positions [e(p-1), ep)."""
    B, K, J, V = target_logits.shape
    lib = load()
    ends = (C.c_int * 4)()
    lib.gls_verify_phases.restype = C.c_int
    lib.gls_verify_phases.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int,
                                      C.c_uint32, C.c_void_p]
    n = int(lib.gls_verify_phases(BF16 if target_logits.dtype == torch.bfloat16 else F32,
                                  int(target_logits.stride(1) != 0), B, K, int(L), V, int(spec),
                                  int(flags), ends))
    if n < 0:
        raise GlsError("gls_verify_phases: arguments that the verify call refuses")
    return [int(ends[i]) for i in range(n)]


def draft_verify_workspace_bytes(B, K, L, J, V):
    return int(load().gls_draft_verify_workspace_bytes(int(B), int(K), int(L), int(J), int(V)))


def draft_verify(draft_logits, target_logits, inv_temp=1.0, inv_temp_per_draft=None,
                 inv_temp_target=None, flags=0, seed=0, seq_base=0, seq_ids=None, pos_base=0,
                 spec=4, rounds=10, noise_flags=0, want_scores=True, workspace=None, status=None,
                 out_draft_tokens=None, out_draft_scores=None, out=None):
    """gls_draft_verify: draft_logits [B,K,L,V] and target_logits [B,K,J,V] (J = L+1, or L with
    NO_BONUS) in one call.  Returns (draft tokens [B,K,L], draft scores | None, dict(tokens, tau,
    accept, scores | None)) -- what draft_sample followed by target_sample_verify return."""
    L_ = load()
    B, K, L, V = draft_logits.shape
    J = target_logits.shape[2]
    assert tuple(target_logits.shape) == (B, K, J, V) and J == (L if (flags & NO_BONUS) else L + 1)
    dev = draft_logits.device
    drows, trows = _rows(draft_logits, 3), _rows(target_logits, 3)
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    given = out_draft_tokens, out_draft_scores, *(() if out is None else out.values())
    if out_draft_tokens is None:
        out_draft_tokens = torch.empty((B, K, L), dtype=torch.int32, device=dev)
    if out_draft_scores is None and want_scores:
        out_draft_scores = torch.empty((B, K, L), dtype=torch.float32, device=dev)
    if out is None:
        out = dict(tokens=torch.empty((B, J), dtype=torch.int32, device=dev),
                   tau=torch.empty((B,), dtype=torch.int32, device=dev),
                   accept=torch.empty((B, K, L), dtype=torch.uint8, device=dev),
                   scores=torch.empty((B, J), dtype=torch.float32, device=dev)
                   if want_scores else None)
    workspace = _workspace(workspace, draft_verify_workspace_bytes(B, K, L, J, V), dev)
    itk = None
    if inv_temp_per_draft is not None:
        itk = (C.c_float * K)(*[float(x) for x in inv_temp_per_draft])
    _check(L_.gls_draft_verify(
        C.byref(drows), C.byref(trows), B, K, L, V, float(inv_temp),
        C.cast(itk, C.c_void_p) if itk is not None else None,
        float(inv_temp if inv_temp_target is None else inv_temp_target), C.byref(nz), int(flags),
        _ptr(out_draft_tokens), _ptr(out_draft_scores), _ptr(out["tokens"]), _ptr(out["tau"]),
        _ptr(out["accept"]), _ptr(out.get("scores")), workspace.data_ptr(), workspace.numel(),
        _ptr(status), _stream()))
    _wrote(*given)
    return out_draft_tokens, out_draft_scores, out


def compress_select(enc_logw, dec_logw=None, bins=None, K=None, seed=0, seq_base=0, seq_ids=None,
                    pos_base=0, spec=4, rounds=10, noise_flags=0, want_scores=True, workspace=None,
                    status=None, out=None):
    """enc_logw [B,N], dec_logw [B,K,N] | None, bins uint8 [N] | [B,N] | None.

    Returns dict(enc_index [B], message [B], dec_index [B,K], match [B], scores [B,1+K] | None)."""
    L = load()
    B, N = enc_logw.shape
    dev = enc_logw.device
    erows = _rows(enc_logw, 1)
    drows = None
    if dec_logw is not None:
        assert dec_logw.shape[0] == B and dec_logw.shape[2] == N
        K = dec_logw.shape[1]
        drows = _rows(dec_logw, 2)
    assert K is not None
    bsb = 0
    if bins is not None:
        if bins.dtype != torch.uint8 or not bins.is_contiguous():
            raise GlsError("bins must be contiguous uint8")
        bsb = 0 if bins.dim() == 1 else N
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    given = out
    if out is None:
        out = dict(enc_index=torch.empty((B,), dtype=torch.int32, device=dev),
                   message=torch.empty((B,), dtype=torch.uint8, device=dev),
                   dec_index=torch.full((B, K), -1, dtype=torch.int32, device=dev),
                   match=torch.zeros((B,), dtype=torch.uint8, device=dev),
                   scores=torch.full((B, 1 + K), float("nan"), dtype=torch.float32, device=dev)
                   if want_scores else None)
    need = workspace_bytes(B, K, 1, N)
    workspace = _workspace(workspace, need, dev)
    _check(L.gls_compress_select(
        C.byref(erows), C.byref(drows) if drows is not None else None, _ptr(bins), bsb, B, K, N,
        C.byref(nz), _ptr(out["enc_index"]), _ptr(out["message"]), _ptr(out["dec_index"]),
        _ptr(out["match"]), _ptr(out.get("scores")), workspace.data_ptr(), workspace.numel(),
        _ptr(status), _stream()))
    if given is not None:
        _wrote(*given.values())
    return out


def compress_gaussian_workspace_bytes(B, K, N):
    return int(load().gls_compress_gaussian_workspace_bytes(int(B), int(K), int(N)))


def compress_gaussian(candidates, source, side_info, bins=None, s2_eta=0.5, s2_zeta=0.25,
                      s2_prior=1.0, seed=0, seq_base=0, seq_ids=None, pos_base=0, spec=4, rounds=10,
                      noise_flags=0, want_scores=True, workspace=None, status=None, out=None):
    """gls_compress_gaussian: candidates [N,D], source [B,D], side_info [B,K,D] (fp32, device).

    Returns compress_select's dict plus recon [B,K,D] and sqerr [B,K]."""
    L = load()
    N, D = candidates.shape
    B, K, _ = side_info.shape
    for x in (candidates, source, side_info):
        if not x.is_cuda or x.dtype != torch.float32 or not x.is_contiguous():
            raise GlsError("candidates, source and side_info must be contiguous float32 device tensors")
    assert tuple(source.shape) == (B, D) and tuple(side_info.shape) == (B, K, D)
    dev = candidates.device
    bsb = 0
    if bins is not None:
        if bins.dtype != torch.uint8 or not bins.is_contiguous():
            raise GlsError("bins must be contiguous uint8")
        bsb = 0 if bins.dim() == 1 else N
    nz = _noise(seed, seq_base, seq_ids, pos_base, spec, rounds, noise_flags)
    given = out
    if out is None:
        out = dict(enc_index=torch.empty((B,), dtype=torch.int32, device=dev),
                   message=torch.empty((B,), dtype=torch.uint8, device=dev),
                   dec_index=torch.full((B, K), -1, dtype=torch.int32, device=dev),
                   match=torch.zeros((B,), dtype=torch.uint8, device=dev),
                   scores=torch.full((B, 1 + K), float("nan"), dtype=torch.float32, device=dev)
                   if want_scores else None,
                   recon=torch.empty((B, K, D), dtype=torch.float32, device=dev),
                   sqerr=torch.empty((B, K), dtype=torch.float32, device=dev))
    workspace = _workspace(workspace, compress_gaussian_workspace_bytes(B, K, N), dev)
    _check(L.gls_compress_gaussian(
        candidates.data_ptr(), source.data_ptr(), side_info.data_ptr(), _ptr(bins), bsb, B, K, N, D,
        float(s2_eta), float(s2_zeta), float(s2_prior), C.byref(nz), _ptr(out["enc_index"]),
        _ptr(out["message"]), _ptr(out["dec_index"]), _ptr(out["match"]), _ptr(out.get("scores")),
        _ptr(out.get("recon")), _ptr(out.get("sqerr")), workspace.data_ptr(), workspace.numel(),
        _ptr(status), _stream()))
    if given is not None:
        _wrote(*given.values())
    return out


# ---- operators next to the sampler: log probabilities, embedding lookup, their gradients ----------
# A call on a few rows takes the GPU about 10 us, so the host's share counts.  The usual call (tensors on
# the current device, results made by the call) is made by the compiled module of csrc/torch_calls.cpp;
# what that does not take, wrong arguments among it, comes back as None and goes the general way below it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda i: torch.cuda.current_stream(i).cuda_stream)
_I32, _F32T, _BF16T, _U8 = torch.int32, torch.float32, torch.bfloat16, torch.uint8


def _ready():
    return _lib if _lib is not None else load()


def _fast():
    if _calls is None:
        load()
    return _calls


def _no_tangent(*tensors):
    """The operators have no forward-mode derivative: a result without the tangent would be a wrong one."""
    if getattr(forward_ad, "_current_level", 0) >= 0:  # within torch.autograd.forward_ad.dual_level()
        for t in tensors:
            if isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None:
                raise GlsError("there is no forward-mode derivative: the call takes no tensor with a tangent")


def _done(r):
    """The compiled module's answer: results, or a status code."""
    if r.__class__ is int:
        raise GlsError(status_string(r))
    return r


def _run(dev, fn, *args):
    """fn(*args, stream) on device index dev and its current stream; GlsError unless it returns 0."""
    if torch.cuda.current_device() == dev:
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        raise GlsError(status_string(rc))


def _device(t, name):
    dev = t.get_device()
    if dev < 0:
        raise GlsError("libgls takes device tensors; %s is not one" % name)
    return dev


def _vec(t, name, shape, dtype, dev):
    """Pointer of a contiguous tensor of this shape and type on device dev (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise GlsError("%s must be a contiguous %s tensor of shape %s on the device of the call's other "
                       "tensors (%d)" % (name, dtype, tuple(shape), dev))
    return t.data_ptr()


def _rows4(t, name):
    """gls_rows_t of a [B,K,J,V] tensor with contiguous rows."""
    if t.dtype is _BF16T:
        dt = BF16
    elif t.dtype is _F32T:
        dt = F32
    else:
        raise GlsError("%s must be float32 or bfloat16" % name)
    st = t.stride()
    if len(st) != 4 or (st[3] != 1 and t.shape[3] > 1):
        raise GlsError("%s must be [B,K,J,V] with a contiguous token dimension" % name)
    if max(t.shape[:3]) > 0x7fffffff:  # possible with strides of 0; the library's counts have 32 bits
        raise GlsError("%s has a dimension beyond 32 bits" % name)
    return _Rows(t.data_ptr(), dt, st[0], st[1], st[2])


def _space(workspace, need, like):
    """(pointer, bytes) of the workspace, made here if there is none."""
    if workspace is None:
        workspace = torch.empty(need, dtype=_U8, device=like.device)
        return workspace, workspace.data_ptr(), need
    if workspace.get_device() != like.get_device() or not workspace.is_contiguous():
        raise GlsError("workspace must be a contiguous tensor on the device of the call's other tensors")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _temps(inv_temp_per_draft, K):
    if inv_temp_per_draft is None:
        return None, None
    v = [float(x) for x in inv_temp_per_draft]
    if len(v) != K:
        raise GlsError("inv_temp_per_draft needs one value per draft")
    a = (C.c_float * K)(*v)
    return a, C.cast(a, C.c_void_p)


def _given(tokens, lead, dev):
    """(pointer, G, shape) of int32 tokens [*lead] or [*lead, G]; none: shape [*lead, 0]."""
    if tokens is None:
        return None, 0, lead + (0,)
    shape = tokens.shape
    if shape[:3] != lead or len(shape) > 4:
        raise GlsError("tokens must have shape %s or that with one more dimension" % (lead,))
    if len(shape) == 4 and shape[3] > MAX_GIVEN:
        raise GlsError("at most %d tokens a row" % MAX_GIVEN)
    return _vec(tokens, "tokens", shape, _I32, dev), shape[3] if len(shape) == 4 else 1, shape


def _top(top):
    top = int(top)
    if not 0 <= top <= 256:
        raise GlsError("top must be between 0 and 256")
    return top


def _score_out(out, like, lead, given, M, want_entropy, dev):
    """(outputs, their pointers: log probabilities, lse, lse's tail, entropy, ids, their log probabilities)"""
    if out is None:
        pe = pi = pt = None
        lse = torch.empty(lead, dtype=_F32T, device=like.device)
        lp = torch.empty_like(lse) if given == lead else lse.new_empty(given)
        out = {"logprobs": lp, "lse": lse}
        if want_entropy:
            out["entropy"] = ent = torch.empty_like(lse)
            pe = ent.data_ptr()
        if M:
            out["top_logprobs"] = tlp = lse.new_empty(lead + (M,))
            out["top_ids"] = ids = tlp.new_empty(lead + (M,), dtype=_I32)
            pi, pt = ids.data_ptr(), tlp.data_ptr()
        return out, lp.data_ptr(), lse.data_ptr(), None, pe, pi, pt
    top = lead + (M,)
    return (out, _vec(out["logprobs"], "out['logprobs']", given, _F32T, dev), _vec(out["lse"], "out['lse']", lead, _F32T, dev),
            _vec(out.get("lse_tail"), "out['lse_tail']", lead, _F32T, dev),
            _vec(out.get("entropy"), "out['entropy']", lead, _F32T, dev),
            _vec(out["top_ids"], "out['top_ids']", top, _I32, dev) if M else None,
            _vec(out["top_logprobs"], "out['top_logprobs']", top, _F32T, dev) if M else None)


def token_logprobs_raw(logits, tokens, top=0, inv_temp=1.0, inv_temp_per_draft=None, want_entropy=True,
                       status=None, out=None):
    """gls_token_logprobs: logits [B,K,J,V], tokens int32 [B,K,J] or [B,K,J,G] (None: no tokens).

    Returns dict(logprobs, lse [B,K,J], entropy [B,K,J], top_ids and top_logprobs [B,K,J,top]); entropy
    only if wanted, the alternatives only for top > 0.  Given `out`, its tensors are written (an
    'lse_tail' among them too).  No autograd: see token_logprobs."""
    _no_tangent(logits)
    if out is None and inv_temp_per_draft is None:
        r = (_calls or _fast()).token_logprobs(logits, tokens, top, inv_temp, want_entropy, status)
        if r is not None:
            return _done(r)
    dev = _device(logits, "logits")
    rows = _rows4(logits, "logits")
    B, K, J, V = logits.shape
    lead, M = (B, K, J), _top(top)
    tp, G, given = _given(tokens, lead, dev)
    out, lp, lse, tail, ent, ids, tlp = _score_out(out, logits, lead, given, M, want_entropy, dev)
    keep, itk = _temps(inv_temp_per_draft, K)
    _run(dev, _ready().gls_token_logprobs, rows, B, K, J, V, float(inv_temp), itk, tp, G, M, lp, lse, tail, ent, ids, tlp,
         _vec(status, "status", (1,), _I32, dev))
    _wrote(*out.values())
    return out


def emitted_logprobs(target_logits, tokens, accept, top=0, inv_temp=1.0, flags=0, want_entropy=True,
                     status=None, out=None):
    """gls_emitted_logprobs: the target rows [B,K,J,V] of a verification with the tokens [B,J] and
    accept flags [B,K,L] it returned -> token_logprobs' dict over [B,J], zeros (alternatives -1) at and
    beyond tau.  Not differentiable: logits that require a gradient are refused where one is recorded."""
    _no_tangent(target_logits)
    if isinstance(target_logits, torch.Tensor) and target_logits.requires_grad and torch.is_grad_enabled():
        raise GlsError("emitted_logprobs has no gradient: give it detached logits or call under torch.no_grad()")
    if out is None:
        r = (_calls or _fast()).emitted_logprobs(target_logits, tokens, accept, top, inv_temp, flags, want_entropy, status)
        if r is not None:
            return _done(r)
    dev = _device(target_logits, "target_logits")
    rows = _rows4(target_logits, "target_logits")
    B, K, J, V = target_logits.shape
    L = J if (flags & NO_BONUS) else J - 1
    lead, M = (B, J), _top(top)
    tp = _vec(tokens, "tokens", lead, _I32, dev)
    ap = _vec(accept, "accept", (B, K, L), _U8, dev) if L > 0 else None
    out, lp, lse, _, ent, ids, tlp = _score_out(out, target_logits, lead, lead, M, want_entropy, dev)
    _run(dev, _ready().gls_emitted_logprobs, rows, B, K, L, V, float(inv_temp), tp, ap, int(flags), M, lp, lse, ent, ids, tlp,
         _vec(status, "status", (1,), _I32, dev))
    _wrote(*out.values())
    return out


def token_logprobs_backward(logits, tokens, lse, entropy=None, lse_tail=None, top_ids=None,
                            grad_logprobs=None, grad_lse=None, grad_entropy=None,
                            grad_top_logprobs=None, inv_temp=1.0, inv_temp_per_draft=None,
                            grad_logits=None):
    """gls_token_logprobs_backward: the gradient with respect to the logits, [B,K,J,V] in their type,
    from token_logprobs' inputs and outputs and the gradients of its outputs (each may be None).  No autograd."""
    _no_tangent(logits, lse, entropy, lse_tail, grad_logprobs, grad_lse, grad_entropy, grad_top_logprobs)
    if grad_logits is None and inv_temp_per_draft is None:
        r = (_calls or _fast()).token_logprobs_backward(logits, tokens, lse, entropy, lse_tail, top_ids, grad_logprobs,
                                                        grad_lse, grad_entropy, grad_top_logprobs, inv_temp)
        if r is not None:
            return _done(r)
    dev = _device(logits, "logits")
    rows = _rows4(logits, "logits")
    shape = logits.shape
    B, K, J, V = shape
    lead = (B, K, J)
    tp, G, given = _given(tokens, lead, dev)
    if grad_entropy is not None and entropy is None:
        raise GlsError("grad_entropy needs the forward call's entropy")
    if grad_top_logprobs is not None and top_ids is None:
        raise GlsError("grad_top_logprobs needs the forward call's top_ids")
    if grad_logprobs is not None and tokens is None:
        raise GlsError("grad_logprobs needs the tokens")
    if grad_logits is None:
        grad_logits = torch.empty(shape, dtype=logits.dtype, device=logits.device)
    elif grad_logits.shape != shape or grad_logits.dtype is not logits.dtype or grad_logits.get_device() != dev:
        raise GlsError("grad_logits must have the logits' shape, type and device")
    M = 0 if top_ids is None else _top(top_ids.shape[-1])
    top = lead + (M,)
    keep, itk = _temps(inv_temp_per_draft, K)
    _run(dev, _ready().gls_token_logprobs_backward, rows, B, K, J, V, float(inv_temp), itk, tp, G,
         _vec(top_ids, "top_ids", top, _I32, dev), M, _vec(lse, "lse", lead, _F32T, dev),
         _vec(lse_tail, "lse_tail", lead, _F32T, dev), _vec(entropy, "entropy", lead, _F32T, dev),
         _vec(grad_logprobs, "grad_logprobs", given, _F32T, dev), _vec(grad_lse, "grad_lse", lead, _F32T, dev),
         _vec(grad_entropy, "grad_entropy", lead, _F32T, dev),
         _vec(grad_top_logprobs, "grad_top_logprobs", top, _F32T, dev), _rows4(grad_logits, "grad_logits"))
    _wrote(grad_logits)
    return grad_logits


def _matrix(t, name):
    """(dtype code, row stride) of a 2-d tensor with contiguous rows."""
    if t.dtype is _BF16T:
        dt = BF16
    elif t.dtype is _F32T:
        dt = F32
    else:
        raise GlsError("%s must be float32 or bfloat16" % name)
    st = t.stride()
    if len(st) != 2 or (st[1] != 1 and t.shape[1] > 1):
        raise GlsError("%s must be a matrix with contiguous rows" % name)
    return dt, st[0]


def embed_tokens_raw(table, tokens, scale=1.0, status=None, out=None):
    """gls_embed_tokens: scale * table[tokens] for table [V,D] and int32 tokens of any shape ->
    [*tokens.shape, D]; a token below 0 gives zeros.  No autograd: see embed_tokens."""
    _no_tangent(table)
    if out is None:
        r = (_calls or _fast()).embed_tokens(table, tokens, scale, status)
        if r is not None:
            return _done(r)
    dev = _device(table, "table")
    dt, stride = _matrix(table, "table")
    V, D = table.shape
    lead = tokens.shape
    tp = _vec(tokens, "tokens", lead, _I32, dev)
    N, ostride = tokens.numel(), D
    if out is None:
        out = torch.empty(lead + (D,), dtype=table.dtype, device=table.device)
    else:
        if out.shape != lead + (D,) or out.dtype is not table.dtype or out.get_device() != dev:
            raise GlsError("out must have shape [*tokens.shape, D], the table's type and its device")
        try:
            flat = out.view(N, D)  # rows a constant stride apart
        except RuntimeError:
            raise GlsError("out's rows must be a constant stride apart") from None
        _, ostride = _matrix(flat, "out")
    _run(dev, _ready().gls_embed_tokens, table.data_ptr(), dt, stride, V, D, tp, N, float(scale), out.data_ptr(), ostride,
         _vec(status, "status", (1,), _I32, dev))
    _wrote(out)
    return out


def embed_tokens_backward_workspace_bytes(N, V, D):
    return int(_ready().gls_embed_tokens_backward_workspace_bytes(N, V, D))


def embed_tokens_backward(grad_out, tokens, V, scale=1.0, grad_table=None, accumulate=False,
                          workspace=None, status=None):
    """gls_embed_tokens_backward: grad_out [*tokens.shape, D] -> the gradient of the table, [V,D] in
    grad_out's type unless grad_table (the same type, or float32) is given.  accumulate: added to
    grad_table, whose other rows are not touched.  No autograd."""
    _no_tangent(grad_out, grad_table)
    if grad_table is None and workspace is None and not accumulate:
        r = (_calls or _fast()).embed_tokens_backward(grad_out, tokens, V, scale, status)
        if r is not None:
            return _done(r)
    dev = _device(grad_out, "grad_out")
    lead, shape = tokens.shape, grad_out.shape
    V = int(V)
    N, D = tokens.numel(), shape[-1] if len(shape) else 0
    if shape != lead + (D,):
        raise GlsError("grad_out must have shape [*tokens.shape, D]")
    tp = _vec(tokens, "tokens", lead, _I32, dev)
    flat = grad_out if grad_out.dim() == 2 else grad_out.reshape(N, D)
    if N and (D > 1 and flat.stride(1) != 1 or N > 1 and flat.stride(0) < D):
        flat = flat.contiguous()  # an expanded gradient
    dt, stride = _matrix(flat, "grad_out")
    if grad_table is None:
        if accumulate:
            raise GlsError("accumulate needs a grad_table to add to")
        grad_table = torch.empty((V, D), dtype=grad_out.dtype, device=grad_out.device)
    elif grad_table.shape != (V, D) or grad_table.get_device() != dev:
        raise GlsError("grad_table must have shape [V, D] and be on grad_out's device")
    gdt, gstride = _matrix(grad_table, "grad_table")
    keep, ws, nbytes = _space(workspace, embed_tokens_backward_workspace_bytes(N, V, D), grad_out)
    _run(dev, _ready().gls_embed_tokens_backward, flat.data_ptr(), dt, stride, tp, N, V, D, float(scale), grad_table.data_ptr(),
         gdt, gstride, EMBED_ACCUMULATE if accumulate else 0, ws, nbytes, _vec(status, "status", (1,), _I32, dev))
    _wrote(grad_table)
    return grad_table


# ---- independent sampling, and a drafter's vocabulary ends at 4 bits -------------------------------
def _no_gradient(name, *tensors):
    if torch.is_grad_enabled():
        for t in tensors:
            if isinstance(t, torch.Tensor) and t.requires_grad:
                raise GlsError("%s has no gradient: give it detached tensors or call under torch.no_grad()" % name)


def _setting(s, name, value, dtype, lead, dev):
    """Puts one sampling setting, a number or a tensor [B], [B,K] or [B,K,J] (sizes of 1 broadcast), into s."""
    if not isinstance(value, torch.Tensor):
        if dtype is not _I32:
            try:
                setattr(s, name, float(value))
            except OverflowError:
                raise GlsError("%s is beyond fp32's range" % name) from None
            if name == "inv_temp" and math.isinf(s.inv_temp) and not math.isinf(value):  # infinity is a setting of its own
                raise GlsError("inv_temp is beyond fp32's range")
        elif value != value or value in (float("inf"), -float("inf")) or int(value) != value:
            raise GlsError("%s must be a whole number" % name)
        else:
            setattr(s, name, max(-1, min(int(value), 2 ** 31 - 1)))  # neither end restricts
        return
    n = value.dim()
    if value.dtype is not dtype or value.get_device() != dev or not 1 <= n <= 3 or any(
            a != b and a != 1 for a, b in zip(value.shape, lead)):
        raise GlsError("%s must be a number or a %s tensor of shape [B], [B,K] or [B,K,J] on the logits' device" % (name, dtype))
    setattr(s, name + "_rows", value.data_ptr())
    st = [value.stride(i) if i < n and value.shape[i] > 1 else 0 for i in range(3)]
    setattr(s, name + "_stride", (C.c_int64 * 3)(*st))


def sample_tokens(logits, uniforms, inv_temp=1.0, top_k=0, top_p=1.0, min_p=0.0, want_logprobs=True, status=None,
                  out=None):
    """gls_sample_tokens: logits [B,K,J,V] and uniforms fp32 [B,K,J] -> dict(tokens int32 [B,K,J], logprobs fp32
    [B,K,J] if wanted), independently per row.

    Each setting is a number or a tensor with a value per sequence [B], or [B,K], or [B,K,J].  inv_temp = inf
    takes the most likely token, top_k < 1 and top_p = 1 and min_p = 0 do not restrict.  Given `out`, its
    tensors are written (log probabilities where it has them).  Not differentiable (see token_logprobs)."""
    _no_tangent(logits, inv_temp, top_p, min_p)
    _no_gradient("sample_tokens", logits, inv_temp, top_p, min_p)
    if out is None:
        r = (_calls or _fast()).sample_tokens(logits, uniforms, inv_temp, top_k, top_p, min_p, want_logprobs, status)
        if r is not None:
            return _done(r)
    dev = _device(logits, "logits")
    rows = _rows4(logits, "logits")
    B, K, J, V = logits.shape
    lead = (B, K, J)
    s = _Sampling()
    _setting(s, "inv_temp", inv_temp, _F32T, lead, dev)
    _setting(s, "top_k", top_k, _I32, lead, dev)
    _setting(s, "top_p", top_p, _F32T, lead, dev)
    _setting(s, "min_p", min_p, _F32T, lead, dev)
    up = _vec(uniforms, "uniforms", lead, _F32T, dev)
    if out is None:
        out = {"tokens": torch.empty(lead, dtype=_I32, device=logits.device)}
        if want_logprobs:
            out["logprobs"] = torch.empty(lead, dtype=_F32T, device=logits.device)
    _run(dev, _ready().gls_sample_tokens, rows, B, K, J, V, s, up, _vec(out["tokens"], "out['tokens']", lead, _I32, dev),
         _vec(out.get("logprobs"), "out['logprobs']", lead, _F32T, dev), _vec(status, "status", (1,), _I32, dev))
    _wrote(*out.values())
    return out


_TYPE_CODE = {_F32T: F32, _BF16T: BF16}


class Int4Table(NamedTuple):
    """A table [V,dim] at 4 bits: codes uint8 [V, at least ceil(dim / 32) * 16], the even column in a byte's low half,
    scales [V, ceil(dim / group)] fp32 or bf16, zeros uint8 of the same shape or None (8).  See gls_int4_table_t."""
    codes: torch.Tensor
    scales: torch.Tensor
    zeros: Optional[torch.Tensor]
    dim: int
    group: int


def _int4(table):
    """(gls_int4_table_t, device index, V) of an Int4Table."""
    codes, scales, zeros, D, group = table
    dev = _device(codes, "codes")
    V, G = codes.shape[0], -(-D // group) if group > 0 else 0
    if codes.dtype is not _U8 or codes.dim() != 2 or (codes.stride(1) != 1 and codes.shape[1] > 1) or codes.shape[1] < -(-D // 32) * 16:
        raise GlsError("codes must be uint8 [V, ceil(dim / 32) * 16] with contiguous rows")
    for t, name in ((scales, "scales"), (zeros, "zeros")):
        if t is not None and (t.shape != (V, G) or t.get_device() != dev or (t.stride(1) != 1 and G > 1)):
            raise GlsError("%s must be [V, ceil(dim / group)] with contiguous rows on the codes' device" % name)
    if zeros is not None and zeros.dtype is not _U8:
        raise GlsError("zeros must be uint8")
    if scales.dtype is not _F32T and scales.dtype is not _BF16T:
        raise GlsError("scales must be float32 or bfloat16")
    return _Int4(codes.data_ptr(), codes.stride(0), scales.data_ptr(), F32 if scales.dtype is _F32T else BF16, scales.stride(0),
                 None if zeros is None else zeros.data_ptr(), 0 if zeros is None else zeros.stride(0), V, D, group), dev, V


def quantize_table(weights, group=128, zeros=True, scale_dtype=torch.bfloat16, out=None):
    """gls_quantize_table: weights [V,D] fp32 or bf16 -> Int4Table with a scale (and a zero) per `group` columns.

    Given `out`, an Int4Table of these sizes, its tensors are written.  Not differentiable."""
    _no_tangent(weights)
    _no_gradient("quantize_table", weights)
    dev = _device(weights, "weights")
    dt, stride = _matrix(weights, "weights")
    V, D = weights.shape
    if out is None:
        if group not in (32, 64, 128):
            raise GlsError("group must be 32, 64 or 128")
        if scale_dtype is not _F32T and scale_dtype is not _BF16T:
            raise GlsError("scale_dtype must be float32 or bfloat16")
        new, G = dict(device=weights.device), -(-D // group)
        out = Int4Table(torch.empty((V, -(-D // 32) * 16), dtype=_U8, **new), torch.empty((V, G), dtype=scale_dtype, **new),
                        torch.empty((V, G), dtype=_U8, **new) if zeros else None, D, group)
    t, tdev, tv = _int4(out)
    if (tv, out.dim, tdev) != (V, D, dev):
        raise GlsError("out must have the weights' sizes and device")
    _run(dev, _ready().gls_quantize_table, weights.data_ptr(), dt, stride, t)
    _wrote(out.codes, out.scales, out.zeros)
    return out


def head_logits_workspace_bytes(N, D, dtype):
    return int(_ready().gls_head_logits_workspace_bytes(int(N), int(D), _TYPE_CODE[dtype]))


def head_logits(x, table, dtype=None, workspace=None, out=None):
    """gls_head_logits: x [...,D] fp32 or bf16 times the rows of an Int4Table [V,D] -> logits [...,V] of type `dtype`
    (x's unless given), accumulated in fp32.  Not differentiable."""
    _no_tangent(x, table.scales)
    _no_gradient("head_logits", x, table.scales)
    if out is None and workspace is None and (dtype is None or dtype in _TYPE_CODE):
        r = (_calls or _fast()).head_logits(x, *table, -1 if dtype is None else _TYPE_CODE[dtype])
        if r is not None:
            return _done(r)
    dev = _device(x, "x")
    t, tdev, V = _int4(table)
    lead = x.shape[:-1]
    if x.dim() < 1 or x.shape[-1] != table.dim or tdev != dev:
        raise GlsError("x must be [..., dim] on the table's device")
    N = lead.numel()
    try:
        flat = x.view(N, table.dim)
    except RuntimeError:
        flat = x.reshape(N, table.dim)
    if N > 1 and flat.stride(0) < table.dim:  # an expanded tensor
        flat = flat.contiguous()
    dt, stride = _matrix(flat, "x")
    if out is None:
        out = torch.empty(lead + (V,), dtype=x.dtype if dtype is None else dtype, device=x.device)
        ostride = V
        odt = _matrix(out.view(N, V), "dtype")[0]
    else:
        if out.shape != lead + (V,) or out.get_device() != dev or (dtype is not None and out.dtype is not dtype):
            raise GlsError("out must have shape [..., V] and be on x's device")
        try:
            odt, ostride = _matrix(out.view(N, V), "out")
        except RuntimeError as e:
            raise e if isinstance(e, GlsError) else GlsError("out's rows must be a constant stride apart") from None
    keep, ws, nbytes = _space(workspace, int(_ready().gls_head_logits_workspace_bytes(N, table.dim, dt)), x)
    _run(dev, _ready().gls_head_logits, flat.data_ptr(), dt, stride, N, t, out.data_ptr(), odt, ostride, ws, nbytes)
    _wrote(out)
    return out


def embed_tokens_int4(table, tokens, scale=1.0, dtype=torch.bfloat16, status=None, out=None):
    """gls_embed_tokens_int4: scale * the rows of an Int4Table [V,D] that int32 tokens of any shape name ->
    [*tokens.shape, D] of type `dtype`; a token below 0 gives zeros.  Not differentiable."""
    _no_tangent(table.scales)
    _no_gradient("embed_tokens_int4", table.scales)
    if out is None and dtype in _TYPE_CODE:
        r = (_calls or _fast()).embed_tokens_int4(*table, tokens, scale, _TYPE_CODE[dtype], status)
        if r is not None:
            return _done(r)
    t, dev, _ = _int4(table)
    D, lead = table.dim, tokens.shape
    tp = _vec(tokens, "tokens", lead, _I32, dev)
    N = tokens.numel()
    if out is None:
        out = torch.empty(lead + (D,), dtype=dtype, device=tokens.device)
    elif out.shape != lead + (D,) or out.get_device() != dev:
        raise GlsError("out must have shape [*tokens.shape, dim] and be on the table's device")
    try:
        flat = out.view(N, D)  # rows a constant stride apart
    except RuntimeError:
        raise GlsError("out's rows must be a constant stride apart") from None
    odt, ostride = _matrix(flat, "out")
    _run(dev, _ready().gls_embed_tokens_int4, t, tp, N, float(scale), out.data_ptr(), odt, ostride,
         _vec(status, "status", (1,), _I32, dev))
    _wrote(out)
    return out
