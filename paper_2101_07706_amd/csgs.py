"""Thin Python binding of libcsgs.so: argument marshalling only.

Same names as the C entry points in include/csgs.h.  Tensors are torch CUDA
(ROCm) tensors used purely as device memory; every step of the method runs in
the library's HIP kernels.  There is no fallback: if the shared library is
missing the import of any entry point raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcsgs.so")

OK, EINVAL, EWORKSPACE, EUNSUPPORTED, ERANGE, ELAUNCH = 0, -1, -2, -3, -4, -5
ST_CAND_OVERFLOW, ST_BAD_EDGE_VALUE, ST_EMPTY_CANDIDATES, ST_ADJ_OVERFLOW, ST_BAD_NODE_ID = 1, 2, 4, 8, 16
ST_EDGE_OVERFLOW, ST_INTERNAL, ST_NONFINITE_GRAD = 32, 64, 128
F32, BF16 = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_LINEAR, GATE_SIGMOID, GATE_SILU = 0, 1, 2
GRAD_L2, GRAD_L1, GRAD_MAX = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_SIGMOID, ACT_SILU, ACT_GELU = 0, 1, 2, 3, 4
STATE_F32, STATE_8BIT, STATE_FIRST, STATE_SECOND, STATE_BLOCK = 0, 1, 0, 1, 256

EXPORTS = ["csgs_workspace_bytes", "csgs_workspace_clean_bytes", "csgs_workspace_init", "csgs_workspace_wait_limit", "csgs_fixed_point", "csgs_build_probs", "csgs_build_probs_auto",
           "csgs_sample_layer", "csgs_draw_nodes", "csgs_sampled_adjacency", "csgs_remote_count", "csgs_aggregate", "csgs_gather_rows",
           "csgs_layer_gemm", "csgs_aggregate_n", "csgs_gather_rows_n", "csgs_layer_gemm_n", "csgs_layer_forward", "csgs_layer_forward_n", "csgs_layer_forward_supported", "csgs_layer_gemm_grad_w_scratch_bytes", "csgs_layer_gemm_grad_w", "csgs_layer_gemm_grad_w_static", "csgs_layer_gemm_grad_z",
           "csgs_aggregate_grad_scratch_bytes", "csgs_aggregate_grad", "csgs_strerror",
           "csgs_embed", "csgs_embed_grad_scratch_bytes", "csgs_embed_grad", "csgs_embed_grad_rows", "csgs_norm_residual",
           "csgs_norm_residual_grad_scratch_bytes", "csgs_norm_residual_grad", "csgs_grad_list_bytes", "csgs_grad_list_init", "csgs_grad_norm",
           "csgs_grad_scale", "csgs_grad_clip", "csgs_adamw_list_bytes", "csgs_adamw_list_init", "csgs_adamw", "csgs_state_read", "csgs_state_write",
           "csgs_linear", "csgs_linear_grad_scratch_bytes", "csgs_linear_grad", "csgs_gated", "csgs_gated_grad_scratch_bytes", "csgs_gated_grad",
           "csgs_profile_enable", "csgs_profile_kernel_count", "csgs_profile_kernel_name", "csgs_profile_collect", "csgs_profile_samples",
           "csgs_calib_copy", "csgs_calib_atomics", "csgs_calib_mfma_f64", "csgs_calib_lookups"]


class CsgsError(RuntimeError):
    def __init__(self, code, where):
        super().__init__(f"{where}: {strerror(code)} ({code})")
        self.code = code


class Graph(C.Structure):
    """csgs_graph: host struct of device pointers."""
    _fields_ = [("n_nodes", C.c_int64), ("nnz", C.c_int64), ("rowptr", C.c_void_p),
                ("colidx", C.c_void_p), ("val", C.c_void_p), ("local_lo", C.c_int32),
                ("local_hi", C.c_int32), ("rownorm2_max", C.c_float)]


class Workspace(C.Structure):
    """csgs_workspace: host descriptor of the caller-owned scratch buffer."""
    _fields_ = [("base", C.c_void_p), ("bytes", C.c_size_t), ("n_nodes", C.c_int64),
                ("nS_max", C.c_int32), ("B_max", C.c_int32), ("edges_max", C.c_int64), ("rows_buf", C.c_uint64),
                ("has_draw", C.c_uint64), ("draw_B", C.c_int32), ("has_next", C.c_int32),
                ("n_inst", C.c_int32), ("scan_mode", C.c_int32), ("inst_stride", C.c_int64)]


class InstStrides(C.Structure):
    """csgs_inst_strides: byte strides between the instances of the _n compute calls."""
    _fields_ = [("n_inst", C.c_int32), ("reserved", C.c_int32), ("adj", C.c_int64), ("x", C.c_int64),
                ("x_remote", C.c_int64), ("out", C.c_int64)]


class RemoteOut(C.Structure):
    """csgs_remote_out: where csgs_sample_layer leaves the remote split of the new node set."""
    _fields_ = [("local_lo", C.c_int32), ("local_hi", C.c_int32), ("part_bounds", C.c_void_p), ("P", C.c_int32),
                ("remote_total", C.c_void_p), ("per_part", C.c_void_p), ("src_row", C.c_void_p),
                ("remote_ids", C.c_void_p)]


class ProbStats(C.Structure):
    """csgs_prob_stats as laid out on the device (64 bytes)."""
    _fields_ = [("n_cand", C.c_int64), ("n_local", C.c_int64), ("n_remote", C.c_int64),
                ("edges_scanned", C.c_int64), ("w_local", C.c_uint64), ("w_remote", C.c_uint64),
                ("total", C.c_uint64), ("shift", C.c_int32), ("skew_fx", C.c_int32)]


class Residual(C.Structure):
    """csgs_residual: host struct of the inputs of csgs_norm_residual and its gradient."""
    _fields_ = [("M", C.c_int32), ("F", C.c_int32), ("M_dev", C.c_void_p), ("x", C.c_void_p), ("h", C.c_void_p), ("gate", C.c_void_p),
                ("ldx", C.c_int64), ("ldh", C.c_int64), ("ldg", C.c_int64), ("post_w", C.c_void_p), ("post_b", C.c_void_p),
                ("pre_w", C.c_void_p), ("pre_b", C.c_void_p), ("x_dtype", C.c_int32), ("h_dtype", C.c_int32), ("post", C.c_int32),
                ("pre", C.c_int32), ("gate_act", C.c_int32), ("eps", C.c_float), ("alpha", C.c_float), ("beta", C.c_float)]


class GradTensor(C.Structure):
    """csgs_grad_tensor: one gradient of a list."""
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ldg", C.c_int64), ("ldo", C.c_int64),
                ("rows_dev", C.c_void_p), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class GradList(C.Structure):
    """csgs_grad_list: host descriptor of a prepared list of gradients."""
    _fields_ = [("base", C.c_void_p), ("bytes", C.c_size_t), ("tiles", C.c_int64), ("n", C.c_int32), ("ready", C.c_int32)]


class LinearArgs(C.Structure):
    """csgs_linear_args: host struct of the inputs of csgs_linear and its gradient."""
    _fields_ = [("M", C.c_int32), ("K", C.c_int32), ("N", C.c_int32), ("act", C.c_int32), ("M_dev", C.c_void_p), ("a", C.c_void_p), ("w", C.c_void_p),
                ("bias", C.c_void_p), ("r", C.c_void_p), ("lda", C.c_int64), ("ldw", C.c_int64), ("ldr", C.c_int64), ("dtype", C.c_int32), ("y_dtype", C.c_int32),
                ("alpha", C.c_float), ("beta", C.c_float)]


class GatedArgs(C.Structure):
    """csgs_gated_args: host struct of the inputs of csgs_gated and its gradient."""
    _fields_ = [("M", C.c_int32), ("K", C.c_int32), ("N", C.c_int32), ("act", C.c_int32), ("M_dev", C.c_void_p), ("x", C.c_void_p), ("wg", C.c_void_p),
                ("wu", C.c_void_p), ("bg", C.c_void_p), ("bu", C.c_void_p), ("ldx", C.c_int64), ("ldwg", C.c_int64), ("ldwu", C.c_int64), ("dtype", C.c_int32),
                ("reserved", C.c_int32)]


class AdamwTensor(C.Structure):
    """csgs_adamw_tensor: one parameter of a list."""
    _fields_ = [("p", C.c_void_p), ("copy", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("ids", C.c_void_p), ("n_dev", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("n", C.c_int64), ("ldp", C.c_int64), ("ldcopy", C.c_int64),
                ("ldg", C.c_int64), ("p_dtype", C.c_int32), ("g_dtype", C.c_int32), ("state", C.c_int32), ("weight_decay", C.c_float), ("lr_scale", C.c_float),
                ("reserved", C.c_int32)]


class AdamwList(C.Structure):
    """csgs_adamw_list: host descriptor of a prepared list of parameters."""
    _fields_ = [("base", C.c_void_p), ("bytes", C.c_size_t), ("tiles", C.c_int64), ("n", C.c_int32), ("ready", C.c_int32)]


class AdamwArgs(C.Structure):
    """csgs_adamw_args: what a step takes beside the list."""
    _fields_ = [("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("lr", C.c_float), ("max_norm", C.c_float), ("lr_dev", C.c_void_p),
                ("step", C.c_void_p), ("clip", C.POINTER(GradList)), ("total", C.c_void_p), ("kind", C.c_int32), ("reserved", C.c_int32), ("norm", C.c_void_p),
                ("status", C.c_void_p)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64, u32, f32, sz = (C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_uint32,
                                           C.c_float, C.c_size_t)
        L.csgs_workspace_bytes.restype = sz
        L.csgs_workspace_bytes.argtypes = [i64, i32, i32, i64]
        L.csgs_workspace_clean_bytes.restype = sz
        L.csgs_workspace_clean_bytes.argtypes = [i64]
        L.csgs_workspace_init.argtypes = [C.POINTER(Workspace), vp]
        L.csgs_workspace_wait_limit.argtypes = [C.POINTER(Workspace), i64, vp]
        L.csgs_fixed_point.argtypes = [i32, f32, f32, C.POINTER(i32), C.POINTER(i64)]
        L.csgs_build_probs.argtypes = [C.POINTER(Graph), vp, i32, vp, f32, vp, vp, vp, vp, i64, vp, C.POINTER(Workspace), vp, vp]
        L.csgs_build_probs_auto.argtypes = [C.POINTER(Graph), vp, i32, vp, f32, i32, f32, vp, vp, vp, vp, i64, vp,
                                            C.POINTER(Workspace), vp, vp]
        L.csgs_sample_layer.argtypes = [C.POINTER(Graph), vp, i32, vp, vp, i64, vp, i32, u64, u64, vp, u32,
                                        vp, vp, vp, vp, vp, vp, vp, i64, vp, C.POINTER(RemoteOut), C.POINTER(Workspace), vp, vp]
        L.csgs_draw_nodes.argtypes = [i64, vp, vp, i64, vp, i32, u64, u64, vp, u32, vp, vp, vp, vp, C.POINTER(Workspace), vp, vp]
        L.csgs_sampled_adjacency.argtypes = [C.POINTER(Graph), vp, i32, vp, vp, vp, vp, i64, vp, C.POINTER(Workspace), vp, vp]
        L.csgs_remote_count.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, vp, vp, vp]
        L.csgs_aggregate.argtypes = [vp, vp, vp, i32, vp, vp, vp, i64, i64, vp, i64, i64, vp, i32, C.c_int,
                                     C.c_int, vp, i64, vp]
        L.csgs_layer_gemm.argtypes = [vp, i64, i32, vp, i32, vp, i64, i32, vp, i64, vp]
        L.csgs_gather_rows.argtypes = [vp, i64, i64, i32, C.c_int, vp, i64, vp, vp, i64, vp]
        strides = [C.POINTER(InstStrides)]
        L.csgs_aggregate_n.argtypes = strides + L.csgs_aggregate.argtypes
        L.csgs_layer_gemm_n.argtypes = strides + L.csgs_layer_gemm.argtypes
        L.csgs_gather_rows_n.argtypes = strides + L.csgs_gather_rows.argtypes
        fwd = [vp, vp, vp, i32, vp, vp, vp, i64, i64, vp, i64, i64, vp, i32, C.c_int, C.c_int, vp, i64, i32, vp, i64, vp, i64]
        L.csgs_layer_forward.argtypes = fwd + [vp]
        L.csgs_layer_forward_n.argtypes = strides + fwd + [i64, vp]
        L.csgs_layer_forward_supported.argtypes = [i32, C.c_int, i64, i64]
        L.csgs_layer_gemm_grad_w_scratch_bytes.restype = sz
        L.csgs_layer_gemm_grad_w_scratch_bytes.argtypes = [i32, i32, i32]
        L.csgs_layer_gemm_grad_w.argtypes = [vp, i64, vp, i64, i32, vp, i32, i32, vp, i64, vp, sz, vp]
        L.csgs_layer_gemm_grad_w_static.argtypes = [vp, i64, vp, i64, i32, vp, i32, i32, vp, i64, vp]
        L.csgs_layer_gemm_grad_z.argtypes = [vp, i64, i32, vp, i32, vp, i64, i32, vp, i64, vp]
        L.csgs_aggregate_grad_scratch_bytes.restype = sz
        L.csgs_aggregate_grad_scratch_bytes.argtypes = [i32, i64]
        L.csgs_aggregate_grad.argtypes = [vp, vp, vp, i64, i32, vp, i32, vp, vp, i64, i32, vp, i64, vp, i64, vp, sz, vp]
        L.csgs_embed.argtypes = [vp, i64, i64, i32, C.c_int, vp, i64, vp, f32, vp, i64, C.c_int, vp]
        L.csgs_embed_grad_scratch_bytes.restype = sz
        L.csgs_embed_grad_scratch_bytes.argtypes = [i64, i64, i32]
        L.csgs_embed_grad.argtypes = [vp, i64, vp, vp, i64, i32, C.c_int, f32, C.c_int, vp, i64, i64, C.c_int, vp, sz, vp]
        L.csgs_embed_grad_rows.argtypes = [vp, i64, vp, vp, i64, i32, C.c_int, f32, i64, vp, vp, vp, i64, C.c_int, vp, sz, vp]
        L.csgs_norm_residual.argtypes = [vp, vp, i64, vp, i64, vp]
        L.csgs_norm_residual_grad_scratch_bytes.restype = sz
        L.csgs_norm_residual_grad_scratch_bytes.argtypes = [i32, i32]
        L.csgs_norm_residual_grad.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, sz, vp]
        L.csgs_grad_list_bytes.restype = sz
        L.csgs_grad_list_bytes.argtypes = [C.POINTER(GradTensor), i32]
        L.csgs_grad_list_init.argtypes = [C.POINTER(GradList), C.POINTER(GradTensor), i32, vp]
        L.csgs_grad_norm.argtypes = [C.POINTER(GradList), C.c_int, vp, vp]
        L.csgs_grad_scale.argtypes = [C.POINTER(GradList), C.c_int, vp, f32, vp, vp, vp]
        L.csgs_grad_clip.argtypes = [C.POINTER(GradList), C.c_int, f32, vp, vp, vp]
        L.csgs_adamw_list_bytes.restype = sz
        L.csgs_adamw_list_bytes.argtypes = [C.POINTER(AdamwTensor), i32]
        L.csgs_adamw_list_init.argtypes = [C.POINTER(AdamwList), C.POINTER(AdamwTensor), i32, vp]
        L.csgs_adamw.argtypes = [C.POINTER(AdamwList), C.POINTER(AdamwArgs), vp]
        L.csgs_state_read.argtypes = [vp, vp, C.c_int, i64, i64, vp, i64, vp]
        L.csgs_state_write.argtypes = [vp, i64, C.c_int, i64, i64, vp, vp, vp]
        L.csgs_linear.argtypes = [vp, vp, i64, vp]
        L.csgs_linear_grad_scratch_bytes.restype = sz
        L.csgs_linear_grad_scratch_bytes.argtypes = [i32, i32, i32, C.c_int]
        L.csgs_linear_grad.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, vp, i64, vp, sz, vp]
        L.csgs_gated.argtypes = [vp, vp, i64, vp]
        L.csgs_gated_grad_scratch_bytes.restype = sz
        L.csgs_gated_grad_scratch_bytes.argtypes = [i32, i32, i32, C.c_int]
        L.csgs_gated_grad.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.csgs_strerror.restype = C.c_char_p
        L.csgs_strerror.argtypes = [C.c_int]
        L.csgs_calib_copy.argtypes = [vp, vp, sz, vp]
        L.csgs_calib_lookups.argtypes = [vp, sz, sz, vp, sz, vp]
        L.csgs_calib_atomics.argtypes = [vp, sz, sz, vp]
        L.csgs_calib_mfma_f64.argtypes = [vp, sz, i64, i32, vp]
        L.csgs_profile_enable.argtypes = [C.c_int]
        L.csgs_profile_kernel_name.restype = C.c_char_p
        L.csgs_profile_kernel_name.argtypes = [C.c_int]
        L.csgs_profile_collect.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.csgs_profile_samples.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_int32), i64, C.POINTER(i64)]
        for name in EXPORTS:
            fn = getattr(L, name)
            # without declared argument types ctypes would pass Python integers as 32-bit values, whose
            # upper half is undefined once they travel on the stack into a 64-bit parameter
            assert fn.argtypes is not None or name in ("csgs_profile_kernel_count",), f"{name}: argument types not declared"
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().csgs_strerror(code).decode()


# A step of a small mini-batch is as long as the host takes to issue it (two-layer steps of 1024 and 777 rows through the helpers of
# pipeline.py, us: 133 and 138 with a ctypes object per pointer, a Stream object per call and a view of the row pointers per
# layer, 119 and 114 -- about the device's time -- without).  Declared argument types turn plain integers into pointers.
def _ptr(t):
    """Device address of a tensor; ctypes objects (a caller's mutable pointer box) pass through."""
    if t is None:
        return None
    if isinstance(t, C._SimpleCData):
        return t
    return t.data_ptr()


_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    """Handle of a stream; None: the current device's current stream."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_device())
    return torch.cuda.current_stream().cuda_stream


def _chk(rc, where):
    if rc != OK:
        raise CsgsError(rc, where)


class DevicePtr(C.c_void_p):
    """A device pointer whose value may be changed between runs of a Plan: stands for an array of
    `n` elements wherever a wrapper takes a tensor only for its address and element count."""

    def __init__(self, n, value=None):
        super().__init__(value)
        self.n = n

    def numel(self):
        return self.n


class Plan:
    """Library calls with their arguments already marshalled, to be issued again and again: a serving
    or training loop that repeats the same calls on the same buffers pays the Python-side marshalling
    once.  Arguments that change between runs are passed as ctypes boxes (c_uint64, c_void_p ...) whose
    value is read at every run.  Built with `with csgs.record() as plan:` around ordinary wrapper calls
    (nothing is enqueued while recording); `plan.run()` enqueues them."""

    def __init__(self):
        self.calls = []

    def run(self):
        for fn, args, name in self.calls:
            rc = fn(*args)
            if rc != OK:
                raise CsgsError(rc, name)


_recording = None


class record:
    def __enter__(self):
        global _recording
        assert _recording is None, "csgs.record() does not nest"
        _recording = Plan()
        return _recording

    def __exit__(self, *exc):
        global _recording
        _recording = None
        return False


def _call(name, *args):
    fn = getattr(lib(), name)
    if _recording is not None:
        _recording.calls.append((fn, args, name))
        return
    _chk(fn(*args), name)


def make_graph(rowptr, colidx, val, local_lo, local_hi, rownorm2_max=1.0) -> Graph:
    assert rowptr.dtype == torch.int64 and colidx.dtype == torch.int32 and val.dtype == torch.float32
    g = Graph(rowptr.numel() - 1, colidx.numel(), rowptr.data_ptr(), colidx.data_ptr(), val.data_ptr(),
              local_lo, local_hi, rownorm2_max)
    g._keep = (rowptr, colidx, val)
    return g


def csgs_workspace_bytes(n_nodes, nS_max, B_max, edges_max) -> int:
    return int(lib().csgs_workspace_bytes(n_nodes, nS_max, B_max, edges_max))


def csgs_workspace_clean_bytes(n_nodes) -> int:
    return int(lib().csgs_workspace_clean_bytes(n_nodes))


def make_workspace(buf, n_nodes, nS_max, B_max, edges_max, n_inst=1, inst_stride=0, scan_mode=0) -> Workspace:
    """Descriptor for `buf` (a torch tensor of at least n_inst * csgs_workspace_bytes(...) bytes).
    n_inst > 1: calls through it process that many instances, whose arrays lie inst_stride bytes apart."""
    ws = Workspace(buf.data_ptr(), buf.numel() * buf.element_size(), n_nodes, nS_max, B_max, edges_max, 0, 0, 0, 0,
                   n_inst, scan_mode, inst_stride)
    ws._keep = buf
    return ws


def csgs_workspace_init(ws, stream=None):
    _call("csgs_workspace_init", C.byref(ws), _stream(stream))


def csgs_workspace_wait_limit(ws, polls, stream=None):
    _call("csgs_workspace_wait_limit", C.byref(ws), polls, _stream(stream))


def csgs_fixed_point(nS, skew, rownorm2_max=1.0):
    sh, sfx = C.c_int32(0), C.c_int64(0)
    rc = lib().csgs_fixed_point(nS, skew, rownorm2_max, C.byref(sh), C.byref(sfx))
    return rc, sh.value, sfx.value


def _rows(S, nS):
    """Row capacity of a call: the length of S, or nS when S is None (rows = the latest sampled set)."""
    return S.numel() if S is not None else nS


def csgs_build_probs(g, S, skew, cand_id, cand_w, cdf, q, stats, ws, status, stream=None, nS_dev=None, nS=None):
    """nS_dev: device int32 holding the number of rows of S to use (S.numel() is then the capacity).
    S None: rows = the node set of the latest csgs_sample_layer on `ws`; nS = that call's B."""
    _call("csgs_build_probs", C.byref(g), _ptr(S), _rows(S, nS), _ptr(nS_dev), skew, _ptr(cand_id), _ptr(cand_w), _ptr(cdf),
                                _ptr(q), cand_id.numel(), _ptr(stats), C.byref(ws), _ptr(status), _stream(stream))


def csgs_build_probs_auto(g, S, D, B, skew_max, cand_id, cand_w, cdf, q, stats, ws, status, stream=None,
                          nS_dev=None, nS=None):
    _call("csgs_build_probs_auto", C.byref(g), _ptr(S), _rows(S, nS), _ptr(nS_dev), D, B, skew_max, _ptr(cand_id), _ptr(cand_w),
                                     _ptr(cdf), _ptr(q), cand_id.numel(), _ptr(stats), C.byref(ws), _ptr(status),
                                     _stream(stream))


def csgs_sample_layer(g, S, cand_id, cdf, stats, B, seed, it, layer, S_next, mult, p_incl, n_next,
                      adj_rowptr, adj_col, adj_val, adj_nnz, ws, status, stream=None, iter_dev=None, remote=None, nS=None):
    """iter_dev: device uint64 tensor holding the iteration number (then `it` is ignored).
    remote: a RemoteOut (see make_remote_out): also write the remote split of S_next."""
    _call("csgs_sample_layer", C.byref(g), _ptr(S), _rows(S, nS), _ptr(cand_id), _ptr(cdf), cand_id.numel(),
                                 _ptr(stats), B, seed, it, _ptr(iter_dev), layer, _ptr(S_next), _ptr(mult), _ptr(p_incl),
                                 _ptr(n_next), _ptr(adj_rowptr), _ptr(adj_col), _ptr(adj_val), adj_col.numel(),
                                 _ptr(adj_nnz), None if remote is None else C.byref(remote), C.byref(ws), _ptr(status), _stream(stream))


def make_remote_out(local_lo, local_hi, part_bounds, remote_total, per_part=None, src_row=None, remote_ids=None) -> RemoteOut:
    dp = lambda t: None if t is None else t.data_ptr()
    r = RemoteOut(local_lo, local_hi, dp(part_bounds), 0 if part_bounds is None else part_bounds.numel() - 1, dp(remote_total),
                  dp(per_part), dp(src_row), dp(remote_ids))
    r._keep = (part_bounds, remote_total, per_part, src_row, remote_ids)
    return r


def csgs_draw_nodes(n_nodes, cand_id, cdf, stats, B, seed, it, layer, S_next, mult, p_incl, n_next, ws, status,
                    stream=None, iter_dev=None):
    _call("csgs_draw_nodes", n_nodes, _ptr(cand_id), _ptr(cdf), cand_id.numel(), _ptr(stats), B, seed, it, _ptr(iter_dev), layer,
                               _ptr(S_next), _ptr(mult), _ptr(p_incl), _ptr(n_next), C.byref(ws), _ptr(status),
                               _stream(stream))


def csgs_sampled_adjacency(g, rows, adj_rowptr, adj_col, adj_val, adj_nnz, ws, status, stream=None,
                           n_rows_dev=None):
    _call("csgs_sampled_adjacency", C.byref(g), _ptr(rows), rows.numel(), _ptr(n_rows_dev), _ptr(adj_rowptr), _ptr(adj_col),
                                      _ptr(adj_val), adj_col.numel(), _ptr(adj_nnz), C.byref(ws), _ptr(status),
                                      _stream(stream))


def csgs_remote_count(S_next, n_next, local_lo, local_hi, part_bounds, remote_total, per_part=None,
                      src_row=None, remote_ids=None, stream=None):
    P = 0 if part_bounds is None else part_bounds.numel() - 1
    _call("csgs_remote_count", _ptr(S_next), _ptr(n_next), local_lo, local_hi, _ptr(part_bounds), P,
                                 _ptr(remote_total), _ptr(per_part), _ptr(src_row), _ptr(remote_ids),
                                 _stream(stream))


def _inst(inst):
    """Leading arguments of a compute call: the _n form with its strides, or the plain form."""
    return ("_n", (C.byref(inst),)) if inst is not None else ("", ())


def csgs_aggregate(adj_rowptr, adj_col, adj_val, n_next, X_local, X_remote, src_row, relu_on_input, Z,
                   stream=None, nS_dev=None, inst=None, nS=None):
    """X_* are 2-D float32 tensors or int16/uint16/bfloat16 tensors holding bfloat16 rows.
    inst (InstStrides): several instances per launch; the tensors are instance 0's.
    nS: row capacity, where adj_rowptr holds more than nS + 1 entries."""
    suffix, lead = _inst(inst)
    dtype = F32 if X_local.dtype == torch.float32 else BF16
    rows_l, F = X_local.shape
    rows_r = 0 if X_remote is None else X_remote.shape[0]
    ld_r = 0 if X_remote is None else X_remote.stride(0)
    if X_remote is not None and rows_r == 0:
        X_remote = None
    Xl_ptr = _ptr(X_local) if rows_l > 0 else None
    rows = adj_rowptr.numel() - 1
    if nS is not None and nS < rows:
        rows = nS
    _call("csgs_aggregate" + suffix, *lead, _ptr(adj_rowptr), _ptr(adj_col), _ptr(adj_val), rows,
                              _ptr(nS_dev), _ptr(n_next), Xl_ptr, X_local.stride(0), rows_l, _ptr(X_remote),
                              ld_r, rows_r, _ptr(src_row), F, dtype, 1 if relu_on_input else 0, _ptr(Z),
                              Z.stride(0), _stream(stream))


def csgs_layer_gemm(Z, W, H, stream=None, M_dev=None, inst=None):
    M, K = Z.shape
    K2, N = W.shape
    assert K == K2 and H.shape == (M, N)
    suffix, lead = _inst(inst)
    _call("csgs_layer_gemm" + suffix, *lead, _ptr(Z), Z.stride(0), M, _ptr(M_dev), K, _ptr(W), W.stride(0), N, _ptr(H), H.stride(0),
                               _stream(stream))


def csgs_layer_forward_supported(X_local, X_remote=None) -> bool:
    """Whether csgs_layer_forward takes input rows of this width, type and layout."""
    dtype = F32 if X_local.dtype == torch.float32 else BF16
    ld_r = 0 if X_remote is None else X_remote.stride(0)
    return bool(lib().csgs_layer_forward_supported(X_local.shape[1], dtype, X_local.stride(0), ld_r))


def csgs_layer_forward(adj_rowptr, adj_col, adj_val, n_next, X_local, X_remote, src_row, relu_on_input, W, H,
                       Z=None, stream=None, nS_dev=None, inst=None, z_stride=0):
    """H = (P~ sigma?(X)) W in one kernel; Z (optional) also receives P~ sigma?(X).  Arguments as csgs_aggregate and
    csgs_layer_gemm; z_stride: bytes between the instances' Z when inst is given."""
    dtype = F32 if X_local.dtype == torch.float32 else BF16
    F_in = X_local.shape[1]
    K2, N = W.shape
    assert K2 == F_in and H.shape == (adj_rowptr.numel() - 1, N)
    rows_r = 0 if X_remote is None else X_remote.shape[0]
    ld_r = 0 if X_remote is None else X_remote.stride(0)
    if X_remote is not None and rows_r == 0:
        X_remote = None
    Xl_ptr = _ptr(X_local) if X_local.shape[0] > 0 else None
    args = (_ptr(adj_rowptr), _ptr(adj_col), _ptr(adj_val), adj_rowptr.numel() - 1, _ptr(nS_dev), _ptr(n_next), Xl_ptr,
            X_local.stride(0), X_local.shape[0], _ptr(X_remote), ld_r, rows_r, _ptr(src_row), F_in, dtype,
            1 if relu_on_input else 0, _ptr(W), W.stride(0), N, _ptr(H), H.stride(0), _ptr(Z), 0 if Z is None else Z.stride(0))
    if inst is not None:
        _call("csgs_layer_forward_n", C.byref(inst), *args, z_stride, _stream(stream))
    else:
        _call("csgs_layer_forward", *args, _stream(stream))


def csgs_layer_gemm_grad_w_scratch_bytes(M, K, N) -> int:
    return int(lib().csgs_layer_gemm_grad_w_scratch_bytes(M, K, N))


def csgs_layer_gemm_grad_w(Z, G, dW, scratch, stream=None, M_dev=None):
    """dW [K x N] = Z^T G; scratch: a tensor of at least csgs_layer_gemm_grad_w_scratch_bytes(M, K, N) bytes."""
    M, K = Z.shape
    M2, N = G.shape
    assert M == M2 and dW.shape == (K, N)
    _call("csgs_layer_gemm_grad_w", _ptr(Z), Z.stride(0), _ptr(G), G.stride(0), M, _ptr(M_dev), K, N, _ptr(dW), dW.stride(0),
          _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream))


GRAD_W_STATIC_BYTES = 32 << 20     # CSGS_GRAD_W_STATIC_BYTES


def csgs_layer_gemm_grad_w_static(Z, G, dW, stream=None, M_dev=None):
    """dW [K x N] = Z^T G with the partial sums in the library's own static device buffer (nothing is allocated)."""
    M, K = Z.shape
    M2, N = G.shape
    assert M == M2 and dW.shape == (K, N)
    _call("csgs_layer_gemm_grad_w_static", _ptr(Z), Z.stride(0), _ptr(G), G.stride(0), M, _ptr(M_dev), K, N, _ptr(dW), dW.stride(0),
          _stream(stream))


def csgs_layer_gemm_grad_z(G, W, dZ, stream=None, M_dev=None):
    """dZ [M x K] = G W^T with W [K x N] as in the forward call."""
    M, N = G.shape
    K, N2 = W.shape
    assert N == N2 and dZ.shape == (M, K)
    _call("csgs_layer_gemm_grad_z", _ptr(G), G.stride(0), M, _ptr(M_dev), N, _ptr(W), W.stride(0), K, _ptr(dZ), dZ.stride(0),
          _stream(stream))


def csgs_aggregate_grad_scratch_bytes(n_cols, adj_cap) -> int:
    return int(lib().csgs_aggregate_grad_scratch_bytes(n_cols, adj_cap))


def csgs_aggregate_grad(adj_rowptr, adj_col, adj_val, n_next, dZ, H_prev, dH_prev, scratch, stream=None, nS_dev=None):
    """dH_prev [n_cols x F] = (P~^T dZ) .* [H_prev > 0]; n_cols = dH_prev.shape[0] (capacity), n_next its device count."""
    nS, F = dZ.shape
    n_cols = dH_prev.shape[0]
    assert adj_rowptr.numel() == nS + 1 and dH_prev.shape[1] == F and (H_prev is None or H_prev.shape[1] == F)
    _call("csgs_aggregate_grad", _ptr(adj_rowptr), _ptr(adj_col), _ptr(adj_val), adj_col.numel(), nS, _ptr(nS_dev), n_cols,
          _ptr(n_next), _ptr(dZ), dZ.stride(0), F, _ptr(H_prev), 0 if H_prev is None else H_prev.stride(0), _ptr(dH_prev),
          dH_prev.stride(0), _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream))


def csgs_gather_rows(X, ids, n_dev, out, stream=None, inst=None):
    """out[k] = X[ids[k]] for k < *n_dev (device int64; None = all of ids)."""
    assert X.dtype == out.dtype and X.shape[1] == out.shape[1] and out.shape[0] >= ids.numel()
    dtype = F32 if X.dtype == torch.float32 else BF16
    suffix, lead = _inst(inst)
    _call("csgs_gather_rows" + suffix, *lead, _ptr(X), X.stride(0), X.shape[0], X.shape[1], dtype, _ptr(ids), ids.numel(),
                                _ptr(n_dev), _ptr(out), out.stride(0), _stream(stream))


_ELEM = {torch.float32: F32, torch.bfloat16: BF16}


def _elem(t):
    """CSGS_* type of a tensor's elements."""
    e = _ELEM.get(t.dtype)
    if e is None:
        raise TypeError(f"float32 or bfloat16, not {t.dtype}")
    return e


def _ld(t, cols):
    """Leading dimension of a matrix whose rows are contiguous (what a tensor says of the step between rows it has one of, does not count)."""
    assert t.dim() == 2 and t.shape[1] == cols and (cols == 1 or t.stride(1) == 1), "rows of a matrix, contiguous"
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), cols)


# The calls below describe up to a dozen tensors, and what torch is asked about each of them is the time of a small one: the usual tensor is contiguous
# and takes four questions (us of host time, a Structure per call and strides, types and sizes asked for one by one / this: residual 12.4 / 4.6,
# its gradient 21 / 7.6).
def _mat(t, shape, dtype):
    """Address and leading dimension of a matrix of this shape and type, or of none."""
    if t is None:
        return None, 0
    assert t.dtype is dtype and t.shape == shape, f"{dtype} of shape {tuple(shape)}, not {t.dtype} of shape {tuple(t.shape)}"
    return t.data_ptr(), shape[1] if t.is_contiguous() else _ld(t, shape[1])


def _i32(t):
    if t is None or isinstance(t, C._SimpleCData):
        return t
    assert t.dtype is torch.int32 and (t.is_contiguous() or t.numel() == 1), "int32, contiguous"
    return t.data_ptr()


def _f32(t, n):
    """A contiguous float vector of n entries, or None."""
    if t is None:
        return None
    assert t.dtype is torch.float32 and t.numel() == n and t.is_contiguous(), f"float32, {n} entries, contiguous"
    return t.data_ptr()


def _scratch(t):
    assert t.is_contiguous()
    return t.data_ptr(), t.numel() * t.element_size()


def _rows_of(t, at_least):
    """Address, leading dimension and width of a matrix of at least so many rows."""
    rows, cols = t.shape
    assert rows >= at_least, f"at least {at_least} rows"
    return t.data_ptr(), cols if t.is_contiguous() else _ld(t, cols), cols


def csgs_embed(T, ids, out, scale=1.0, n_dev=None, stream=None):
    """out[t] = scale * T[ids[t]] (float32 or bfloat16 each); zeros where an id is outside the table."""
    n = ids.numel()
    rows, F = T.shape
    op, ldo, cols = _rows_of(out, n)
    assert cols == F, "as wide as the table"
    _call("csgs_embed", T.data_ptr(), F if T.is_contiguous() else _ld(T, F), rows, F, _elem(T), _i32(ids), n, _i32(n_dev), scale, op, ldo, _elem(out),
          _stream(stream))


def csgs_embed_grad_scratch_bytes(n, rows, F) -> int:
    return int(lib().csgs_embed_grad_scratch_bytes(n, rows, F))


def csgs_embed_grad(ids, G, dT, scratch, scale=1.0, accumulate=False, n_dev=None, stream=None):
    """dT[v] = scale * sum of G[t] over ids[t] = v, zeros elsewhere; accumulate: added to what dT holds.
    scratch: a tensor of at least csgs_embed_grad_scratch_bytes(len(ids), len(dT), F) bytes."""
    n = ids.numel()
    gp, ldg, F = _rows_of(G, n)
    rows, cols = dT.shape
    assert cols == F, "as wide as the table"
    ptr, nbytes = _scratch(scratch)
    _call("csgs_embed_grad", _i32(ids), n, _i32(n_dev), gp, ldg, F, _elem(G), scale, 1 if accumulate else 0, dT.data_ptr(),
          F if dT.is_contiguous() else _ld(dT, F), rows, _elem(dT), ptr, nbytes, _stream(stream))


def csgs_embed_grad_rows(ids, G, rows, uniq, n_uniq, dR, scratch, scale=1.0, n_dev=None, stream=None):
    """The rows of that gradient that some id points to alone: uniq ascending, *n_uniq of them, dR[j] the gradient of row uniq[j]."""
    n = ids.numel()
    gp, ldg, F = _rows_of(G, n)
    dp, ldd, cols = _rows_of(dR, n)
    assert cols == F and uniq.numel() >= n, "a row and an id for every position"
    ptr, nbytes = _scratch(scratch)
    _call("csgs_embed_grad_rows", _i32(ids), n, _i32(n_dev), gp, ldg, F, _elem(G), scale, rows, _i32(uniq), _i32(n_uniq), dp, ldd, _elem(dR), ptr, nbytes,
          _stream(stream))


_residual_layout = struct.Struct("<iiQQQQqqqQQQQiiiiifff")     # csgs_residual


def _residual(x, h, stream, block, gate, gate_act, post, post_w, post_b, pre, pre_w, pre_b, eps, alpha, beta, M_dev):
    """csgs_residual, its shape, and the tensors' types; `stream` and `block`: a tensor of each of the two."""
    shape = (x if x is not None else h).shape
    M, F = shape
    ts, tb = stream.dtype, block.dtype
    xp, ldx = _mat(x, shape, ts)
    hp, ldh = _mat(h, shape, tb)
    if gate is None:
        gp, ldg = 0, 0
    elif gate.dim() == 1:
        gp, ldg = _f32(gate, F), 0
    else:
        gp, ldg = _mat(gate, shape, tb)
    if M_dev is not None:
        assert M_dev.dtype is torch.int32
        M_dev = M_dev.data_ptr()
    r = _residual_layout.pack(M, F, M_dev or 0, xp or 0, hp or 0, gp, ldx, ldh, ldg, _f32(post_w, F) or 0, _f32(post_b, F) or 0, _f32(pre_w, F) or 0,
                              _f32(pre_b, F) or 0, _elem(stream), _elem(block), post, pre, gate_act, eps, alpha, beta)
    return r, shape, ts, tb


def csgs_norm_residual(x, h, y, u, gate=None, gate_act=GATE_LINEAR, post=NORM_RMS, post_w=None, post_b=None, pre=NORM_RMS, pre_w=None, pre_b=None,
                       eps=1e-5, alpha=1.0, beta=1.0, M_dev=None, stream=None):
    """y = beta x + alpha a(gate) .* N(h; post_w, post_b), u = N(y; pre_w, pre_b).  x or h, y or u may be None.
    gate: None, a float32 vector for all rows, or a matrix like h."""
    a = x if x is not None else y if y is not None else h     # a tensor of the stream's type, of the block's
    b = h if h is not None else u if u is not None else x
    r, shape, ts, tb = _residual(x, h, a, b, gate, gate_act, post, post_w, post_b, pre, pre_w, pre_b, eps, alpha, beta, M_dev)
    _call("csgs_norm_residual", r, *_mat(y, shape, ts), *_mat(u, shape, tb), _stream(stream))


def csgs_norm_residual_grad_scratch_bytes(M, F) -> int:
    return int(lib().csgs_norm_residual_grad_scratch_bytes(M, F))


def csgs_norm_residual_grad(x, h, dy, du, dx, dh, dgate, dpost_w, dpost_b, dpre_w, dpre_b, scratch, gate=None, gate_act=GATE_LINEAR, post=NORM_RMS,
                            post_w=None, post_b=None, pre=NORM_RMS, pre_w=None, pre_b=None, eps=1e-5, alpha=1.0, beta=1.0, M_dev=None, stream=None):
    """Gradients of csgs_norm_residual from dy and du (one may be None); outputs may be None.
    scratch: a tensor of at least csgs_norm_residual_grad_scratch_bytes(M, F) bytes."""
    a = x if x is not None else dy if dy is not None else dx if dx is not None else h
    b = h if h is not None else du if du is not None else dh if dh is not None else x
    r, shape, ts, tb = _residual(x, h, a, b, gate, gate_act, post, post_w, post_b, pre, pre_w, pre_b, eps, alpha, beta, M_dev)
    F = shape[1]
    dg, lddg = (_f32(dgate, F), 0) if gate is None or gate.dim() == 1 else _mat(dgate, shape, tb)
    ptr, nbytes = _scratch(scratch)
    _call("csgs_norm_residual_grad", r, *_mat(dy, shape, ts), *_mat(du, shape, tb), *_mat(dx, shape, ts), *_mat(dh, shape, tb), dg, lddg, _f32(dpost_w, F),
          _f32(dpost_b, F), _f32(dpre_w, F), _f32(dpre_b, F), ptr, nbytes, _stream(stream))


def _torch_stream(stream):
    """The stream as torch knows it; None: the current one."""
    if stream is None:
        return torch.cuda.current_stream()
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)


def _list_on(l, stream):
    """A list as an argument of a call on `stream`.  Its buffer is no tensor that the caller holds: torch is told, once for every stream that it is used on, not to
    hand the memory out again before what is enqueued there by the time the list is dropped has run."""
    streams = getattr(l, "_streams", None)     # (a list that make_grad_list has not made brings memory of its own)
    if streams is not None:
        handle = _stream(stream)
        if handle not in streams:
            l._keep[0].record_stream(_torch_stream(stream))
            streams.add(handle)
    return C.byref(l)


def _list_buffer(nbytes, device, stream):
    """Memory that this stream's earlier work may still use, and no other's."""
    with torch.cuda.stream(stream if stream is None else _torch_stream(stream)):
        return torch.empty(nbytes // 8, dtype=torch.int64, device=device)


def _as_matrix(t):
    """A tensor as rows x cols."""
    return t if t.dim() == 2 else t.reshape(1, -1) if t.is_contiguous() else t.unsqueeze(0)


def make_grad_list(grads, outs=None, rows_dev=None, stream=None) -> GradList:
    """A list of gradients for csgs_grad_norm / _scale / _clip, described once in device memory.  outs: where the clipped gradients go (None: in
    place; entries may be None); rows_dev: per gradient, a device int32 with the number of rows that count, or None.
    The list keeps the tensors; they must not be resized or freed by other means.  It may be dropped while calls that use it are still enqueued: its own buffer
    comes from the pool of `stream` and is given back when these are done, on whatever streams they are (the gradients are the caller's, as in every call).  A
    plan keeps the list; one that was captured into a graph has to be kept as long as the graph is replayed."""
    outs = grads if outs is None else outs
    rows_dev = [None] * len(grads) if rows_dev is None else rows_dev
    assert len(grads) > 0 and len(outs) == len(grads) and len(rows_dev) == len(grads)
    assert _recording is None, "a list is made once, not by a recorded call"
    matrix = _as_matrix
    ts = (GradTensor * len(grads))()
    for i, (g, o, n) in enumerate(zip(grads, outs, rows_dev)):
        assert o is None or (o.shape == g.shape and o.dtype == g.dtype)
        assert n is None or g.dim() == 2, "rows are those of a matrix"
        m = matrix(g)
        ts[i] = GradTensor(_ptr(g), _ptr(o), m.shape[0], m.shape[1], _ld(m, m.shape[1]), 0 if o is None else _ld(matrix(o), m.shape[1]), _i32(n), _elem(g), 0)
    nbytes = int(lib().csgs_grad_list_bytes(ts, len(grads)))
    if nbytes == 0:
        raise CsgsError(EINVAL, "csgs_grad_list_bytes")
    buf = _list_buffer(nbytes, grads[0].device, stream)
    l = GradList(buf.data_ptr(), nbytes, 0, 0, 0)
    l._keep, l._streams = (buf, list(grads), list(outs), list(rows_dev)), {_stream(stream)}
    _call("csgs_grad_list_init", C.byref(l), ts, len(grads), _stream(stream))
    return l


def csgs_grad_norm(l, kind, total, stream=None):
    """total: float64 tensor of one entry; receives the sum of squares, of absolute values, or the largest of these."""
    assert total.dtype == torch.float64
    _call("csgs_grad_norm", _list_on(l, stream), kind, _ptr(total), _stream(stream))


def csgs_grad_scale(l, kind, total, max_norm, norm=None, status=None, stream=None):
    assert total.dtype == torch.float64
    _call("csgs_grad_scale", _list_on(l, stream), kind, _ptr(total), max_norm, _f32(norm, 1), _i32(status), _stream(stream))


def csgs_grad_clip(l, kind, max_norm, norm=None, status=None, stream=None):
    """out = min(1, max_norm / (total + 1e-6)) g over the list; norm receives the total before clipping."""
    _call("csgs_grad_clip", _list_on(l, stream), kind, max_norm, _f32(norm, 1), _i32(status), _stream(stream))


_linear_layout, _gated_layout = struct.Struct("<iiiiQQQQQqqqiiff"), struct.Struct("<iiiiQQQQQQqqqii")     # csgs_linear_args, csgs_gated_args


def _linear(a, w, y, bias, r, act, alpha, beta, M_dev):
    """csgs_linear_args and the shape of y; y: a tensor of the output's type."""
    M, K = a.shape
    N = w.shape[1]
    ap, lda = _mat(a, (M, K), a.dtype)
    wp, ldw = _mat(w, (K, N), a.dtype)
    rp, ldr = _mat(r, (M, N), y.dtype)
    args = _linear_layout.pack(M, K, N, act, _i32(M_dev) or 0, ap, wp, _f32(bias, N) or 0, rp or 0, lda, ldw, ldr, _elem(a), _elem(y), alpha, beta)
    return args, (M, K, N)


def csgs_linear(a, w, y, bias=None, r=None, act=ACT_NONE, alpha=1.0, beta=1.0, M_dev=None, stream=None):
    """y = alpha act(a w + bias) + beta r.  a and w float32 or bfloat16, bias float32, r and y of their type or, for bfloat16, float32."""
    args, (M, K, N) = _linear(a, w, y, bias, r, act, alpha, beta, M_dev)
    _call("csgs_linear", args, *_mat(y, (M, N), y.dtype), _stream(stream))


def csgs_linear_grad_scratch_bytes(M, K, N, dtype) -> int:
    """dtype: F32 or BF16, of a and w."""
    return int(lib().csgs_linear_grad_scratch_bytes(M, K, N, dtype))


def csgs_linear_grad(a, w, dy, da, dw, dbias, dr, scratch, bias=None, act=ACT_NONE, alpha=1.0, beta=1.0, M_dev=None, stream=None):
    """Gradients of csgs_linear from dy; outputs may be None.  scratch: a tensor of at least csgs_linear_grad_scratch_bytes(M, K, N, dtype) bytes."""
    args, (M, K, N) = _linear(a, w, dy, bias, dr, act, alpha, beta, M_dev)      # (of r only that there is one counts)
    ptr, nbytes = _scratch(scratch)
    _call("csgs_linear_grad", args, *_mat(dy, (M, N), dy.dtype), *_mat(da, (M, K), a.dtype), *_mat(dw, (K, N), a.dtype), _f32(dbias, N), *_mat(dr, (M, N), dy.dtype),
          ptr, nbytes, _stream(stream))


def _gated(x, wg, wu, bg, bu, act, M_dev):
    M, K = x.shape
    N = wg.shape[1]
    xp, ldx = _mat(x, (M, K), x.dtype)
    gp, ldwg = _mat(wg, (K, N), x.dtype)
    up, ldwu = _mat(wu, (K, N), x.dtype)
    return _gated_layout.pack(M, K, N, act, _i32(M_dev) or 0, xp, gp, up, _f32(bg, N) or 0, _f32(bu, N) or 0, ldx, ldwg, ldwu, _elem(x), 0), (M, K, N)


def csgs_gated(x, wg, wu, h, bg=None, bu=None, act=ACT_SILU, M_dev=None, stream=None):
    """h = act(x wg + bg) .* (x wu + bu); x, wg, wu and h float32 or bfloat16, the same for all, bg and bu float32."""
    args, (M, K, N) = _gated(x, wg, wu, bg, bu, act, M_dev)
    _call("csgs_gated", args, *_mat(h, (M, N), x.dtype), _stream(stream))


def csgs_gated_grad_scratch_bytes(M, K, N, dtype) -> int:
    """dtype: F32 or BF16, of x, wg and wu."""
    return int(lib().csgs_gated_grad_scratch_bytes(M, K, N, dtype))


def csgs_gated_grad(x, wg, wu, dh, dx, dwg, dwu, dbg, dbu, scratch, bg=None, bu=None, act=ACT_SILU, M_dev=None, stream=None):
    """Gradients of csgs_gated from dh; outputs may be None.  scratch: a tensor of at least csgs_gated_grad_scratch_bytes(M, K, N, dtype) bytes."""
    args, (M, K, N) = _gated(x, wg, wu, bg, bu, act, M_dev)
    ptr, nbytes = _scratch(scratch)
    _call("csgs_gated_grad", args, *_mat(dh, (M, N), x.dtype), *_mat(dx, (M, K), x.dtype), *_mat(dwg, (K, N), x.dtype), *_mat(dwu, (K, N), x.dtype), _f32(dbg, N),
          _f32(dbu, N), ptr, nbytes, _stream(stream))


def adamw_states(p, bits=32):
    """States of a new parameter, all zero, for adamw_entry: dict of m and v, for bits=8 also of m_exp and v_exp."""
    assert bits in (8, 32)
    rows, cols = _as_matrix(p).shape
    if bits == 32:
        return {k: torch.zeros(rows, cols, dtype=torch.float32, device=p.device) for k in ("m", "v")}
    blocks = (cols + STATE_BLOCK - 1) // STATE_BLOCK
    return {k: torch.zeros(rows, blocks if "exp" in k else cols, dtype=torch.uint8, device=p.device) for k in ("m", "v", "m_exp", "v_exp")}


def _meet(a, b):
    """Whether the memory that two tensors span meets."""
    end = lambda t: t.data_ptr() + (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1) * t.element_size()  # noqa: E731
    return a.data_ptr() < end(b) and b.data_ptr() < end(a)


def adamw_entry(p, g, m, v, m_exp=None, v_exp=None, copy=None, ids=None, n_dev=None, weight_decay=0.0, lr_scale=1.0):
    """A parameter for make_adamw_list: p with its gradient g, states m and v (float32, or uint8 with exponents m_exp and v_exp: adamw_states), a bfloat16
    copy of p, for a table whose gradient holds rows alone their ids (strictly ascending), a device int32 with the number of rows of g that count."""
    mp, mg = _as_matrix(p), _as_matrix(g)
    rows, cols = mp.shape
    n = mg.shape[0]
    assert mg.shape[1] == cols and (ids is not None or n == rows), "a gradient like its parameter, or rows of it with their ids"
    assert ids is None or (p.dim() == 2 and ids.numel() >= n), "an id for every row of the gradient"
    assert n_dev is None or g.dim() == 2, "rows are those of a matrix"
    small = m.dtype is torch.uint8
    for t in (m, v):
        assert t.dtype is (torch.uint8 if small else torch.float32) and t.numel() == rows * cols and t.is_contiguous(), "states like the parameter, contiguous"
    blocks = (cols + STATE_BLOCK - 1) // STATE_BLOCK
    assert (m_exp is None) == (v_exp is None) == (not small), "exponents for states in 8 bits"
    for t in (m_exp, v_exp):
        assert t is None or (t.dtype is torch.uint8 and t.numel() == rows * blocks and t.is_contiguous()), f"uint8, {blocks} a row, contiguous"
        assert t is None or not any(_meet(t, u) for u in (p, g, m, v, copy, m_exp if t is v_exp else v_exp) if u is not None), "exponents in memory of their own"
    ldcopy = 0
    if copy is not None:
        assert copy.dtype is torch.bfloat16 and copy.shape == p.shape, "a bfloat16 copy of the parameter's shape"
        ldcopy = _ld(_as_matrix(copy), cols)
    e = AdamwTensor(_ptr(p), _ptr(copy), _ptr(g), _ptr(m), _ptr(v), _ptr(m_exp), _ptr(v_exp), _i32(ids), _i32(n_dev), rows, cols, n, _ld(mp, cols), ldcopy,
                    _ld(mg, cols), _elem(p), _elem(g), STATE_8BIT if small else STATE_F32, weight_decay, lr_scale, 0)
    e._keep = (p, g, m, v, m_exp, v_exp, copy, ids, n_dev)
    return e


def make_adamw_list(entries, stream=None) -> AdamwList:
    """A list of parameters (adamw_entry) for csgs_adamw, described once in device memory.  The list keeps their tensors, and is kept and dropped as those of
    make_grad_list are."""
    assert len(entries) > 0
    assert _recording is None, "a list is made once, not by a recorded call"
    written = [e._keep[k].data_ptr() for e in entries for k in (0, 2, 3)]
    assert len(set(written)) == len(written), "a parameter and its states belong to one entry"
    ts = (AdamwTensor * len(entries))(*entries)
    nbytes = int(lib().csgs_adamw_list_bytes(ts, len(entries)))
    if nbytes == 0:
        raise CsgsError(EINVAL, "csgs_adamw_list_bytes")
    buf = _list_buffer(nbytes, entries[0]._keep[0].device, stream)
    l = AdamwList(buf.data_ptr(), nbytes, 0, 0, 0)
    l._keep, l._streams = (buf, [e._keep for e in entries]), {_stream(stream)}
    _call("csgs_adamw_list_init", C.byref(l), ts, len(entries), _stream(stream))
    return l


def csgs_adamw(l, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, clip=None, total=None, kind=GRAD_L2, max_norm=float("inf"), lr_dev=None, norm=None, status=None,
               stream=None):
    """One step over a list of make_adamw_list.  step: device int32, the steps taken so far.  clip: a list of make_grad_list whose norm bounds the gradients by
    max_norm (or total: a float64 of csgs_grad_norm); gradients whose norm is not finite change nothing.  lr_dev: a float32 that multiplies lr."""
    assert total is None or total.dtype == torch.float64
    assert step.dtype is torch.int32 and step.numel() == 1
    grads = None
    if clip is not None:
        _list_on(clip, stream)
        grads = C.pointer(clip)
    a = AdamwArgs(beta1, beta2, eps, lr, max_norm, _f32(lr_dev, 1), step.data_ptr(), grads, _ptr(total), kind, 0, _f32(norm, 1), _i32(status))
    _call("csgs_adamw", _list_on(l, stream), C.byref(a), _stream(stream))


def _state_shape(codes, exps):
    rows, cols = _as_matrix(codes).shape
    blocks = (cols + STATE_BLOCK - 1) // STATE_BLOCK
    assert codes.dtype is torch.uint8 and exps.dtype is torch.uint8 and codes.is_contiguous() and exps.is_contiguous() and exps.numel() == rows * blocks
    return rows, cols


def csgs_state_read(codes, exps, which, values, stream=None):
    """The values (float32) of states in 8 bits; which: STATE_FIRST (m) or STATE_SECOND (v)."""
    rows, cols = _state_shape(codes, exps)
    vp, ld = _mat(_as_matrix(values), (rows, cols), torch.float32)
    _call("csgs_state_read", codes.data_ptr(), exps.data_ptr(), which, rows, cols, vp, ld, _stream(stream))


def csgs_state_write(values, which, codes, exps, stream=None):
    """States in 8 bits from their values (float32)."""
    rows, cols = _state_shape(codes, exps)
    vp, ld = _mat(_as_matrix(values), (rows, cols), torch.float32)
    _call("csgs_state_write", vp, ld, which, rows, cols, codes.data_ptr(), exps.data_ptr(), _stream(stream))


def csgs_profile_enable(on: bool):
    _call("csgs_profile_enable", 1 if on else 0)


def csgs_profile_collect():
    """{kernel name: (summed ms, launches)} since the last collect; call after synchronising."""
    n = lib().csgs_profile_kernel_count()
    ms = (C.c_double * n)()
    cnt = (C.c_int64 * n)()
    _call("csgs_profile_collect", ms, cnt)
    return {lib().csgs_profile_kernel_name(k).decode(): (ms[k], cnt[k]) for k in range(n) if cnt[k]}


def csgs_profile_samples(cap=1 << 16):
    """{kernel name: [ms of every launch]} since the last collect (does not reset); call after synchronising."""
    ms = (C.c_float * cap)()
    kid = (C.c_int32 * cap)()
    n = C.c_int64(0)
    _call("csgs_profile_samples", ms, kid, cap, C.byref(n))
    out = {}
    for i in range(min(cap, n.value)):
        if ms[i] >= 0:
            out.setdefault(lib().csgs_profile_kernel_name(kid[i]).decode(), []).append(ms[i])
    return out


def csgs_calib_copy(dst, src, stream=None):
    nbytes = src.numel() * src.element_size()
    _call("csgs_calib_copy", _ptr(dst), _ptr(src), nbytes, _stream(stream))


def csgs_calib_atomics(table, n_updates, stream=None):
    """n_updates atomic +1 on pseudo-random entries of `table` (an int64 tensor)."""
    _call("csgs_calib_atomics", _ptr(table), table.numel(), n_updates, _stream(stream))


def csgs_calib_lookups(table, n_reads, sink, stream=None):
    """n_reads 8-byte reads of pseudo-random entries of `table` (int64 tensor); sink: int64 tensor of >= 4194304 entries."""
    _call("csgs_calib_lookups", _ptr(table), table.numel(), n_reads, _ptr(sink), sink.numel(), _stream(stream))


CALIB_MFMA_BLOCKS = 2048   # CSGS_CALIB_MFMA_BLOCKS


def csgs_calib_mfma_f64(sink, iters, from_lds=False, stream=None):
    """Matrix-core yardstick; returns the flops of the call.  `sink`: float64 tensor of at least
    CALIB_MFMA_BLOCKS * 256 entries."""
    _call("csgs_calib_mfma_f64", _ptr(sink), sink.numel(), iters, 1 if from_lds else 0, _stream(stream))
    return CALIB_MFMA_BLOCKS * 4 * 64 * 2048 * iters
