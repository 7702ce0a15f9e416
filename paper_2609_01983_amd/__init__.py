"""MI355X-native DualGCN aggregation: Python binding of ``libdualgcn.so``.

Argument marshalling only -- every step of the path runs in the library's HIP
kernels.  torch provides device memory and the current stream.  The library is
built by ``python paper_2609_01983_amd/build.py`` (or ``__graft_entry__.build()``); if it
is missing, importing this package raises ImportError: there is no fallback.

    plan = Plan(rowptr, col, val, seed=0, walks_per_node=16, walk_len=5)
    Y = spmm(plan, X)                           # Y = A X
    T = update(X, W)                            # T = X W, bf16 matrix cores
    H = gcn_layer(plan, X, W, relu=True)        # H = relu(A (X W)), X W in bf16 MFMA

Between the blocks of a deep GCN, in training from a teacher, and in serving from 8 bits:

    R, Z = norm_residual(R, B, gate=gate)       # R + gate * norm(B), and its norm
    G, loss = distill_xent(Y, ids, teacher)     # against the teacher's top logits, and dloss/dY
    T = update_fp8(*quantize_fp8(Z), *W8)       # T = Z W, e4m3 with a scale for each 128
    T = update_mxfp4(*quantize_mxfp4(Z), *W4)   # T = Z W, e2m1 with a scale for each 32

Over the graphs of a batch, and for all weights at once:

    Y, stats = group_norm(X, ptr, groups=8, act="silu")    # and group_norm_backward
    norm = clipped_sgd(weights, grads, lr, max_norm=1.0)   # W -= lr * clipped gradient
"""
import array
import collections
import ctypes
import os

import torch  # must load before the library: it provides the process's HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdualgcn.so")

OK, ERR_INVALID_ARG, ERR_BAD_CSR, ERR_UNSUPPORTED, ERR_OOM, ERR_HIP, ERR_NO_DEVICE = \
    0, -1, -2, -3, -4, -5, -6
FORCE_AUTO, FORCE_SPARSE, FORCE_DENSE = 0, 1, 2
RELU, OUT_BF16, IN_BF16, GRAD_BF16 = 1, 2, 4, 8
STREAM_BF16, NORM_LAYER, NORM_POST = 16, 32, 64
GATE_FEATURE, GATE_NODE, GATE_FULL, GATE_SIGMOID = 128, 256, 512, 1024
TEACHER_BF16, SILU, ZERO_REST = 2048, 4096, 8192
FP8_BLOCK = 128                  # elements that share a scale in the 8-bit operands
MX_BLOCK = 32                    # and in the 4-bit ones
LOSS_SLOTS = 1025                # float64 entries of the loss buffer of softmax_xent
ALPHA_ADAPTIVE = 0xFFFFFFFF      # alpha = (ALPHA_ADAPTIVE, q): adaptive weight in steps of 1/q
ALPHA_BALANCED = 0xFFFFFFFE      # alpha = (ALPHA_BALANCED, q): weight balancing the spreads of N and D

_FORCE = {"auto": FORCE_AUTO, "sparse": FORCE_SPARSE, "dense": FORCE_DENSE,
          FORCE_AUTO: FORCE_AUTO, FORCE_SPARSE: FORCE_SPARSE, FORCE_DENSE: FORCE_DENSE}


class DualGCNError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {status_str(status)} ({status})"
                         + (f", hip error {_lib.dualgcn_last_hip_error()}" if status == ERR_HIP else ""))


class Csr(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("nnz", ctypes.c_int64), ("rowptr", ctypes.c_void_p),
                ("col", ctypes.c_void_p), ("val", ctypes.c_void_p)]


class Thresholds(ctypes.Structure):
    _fields_ = [("alpha_num", ctypes.c_uint32), ("alpha_den", ctypes.c_uint32),
                ("beta_num", ctypes.c_uint32), ("beta_den", ctypes.c_uint32),
                ("force_mode", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("nnz", ctypes.c_int64), ("n_sparse", ctypes.c_int32),
                ("n_dense", ctypes.c_int32), ("kstar", ctypes.c_uint64),
                ("s1_hi", ctypes.c_uint64), ("s1_lo", ctypes.c_uint64),
                ("s2_hi", ctypes.c_uint64), ("s2_lo", ctypes.c_uint64), ("kmax", ctypes.c_uint64),
                ("alpha_num", ctypes.c_uint32), ("alpha_den", ctypes.c_uint32),
                ("beta_num", ctypes.c_uint32), ("beta_den", ctypes.c_uint32),
                ("force_mode", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("walks_per_node", ctypes.c_uint32), ("walk_len", ctypes.c_uint32),
                ("max_degree", ctypes.c_int32), ("dense_chunk", ctypes.c_int32),
                ("n_split_rows", ctypes.c_int32), ("n_split_parts", ctypes.c_int32),
                ("n_tasks", ctypes.c_int32), ("n_long_rows", ctypes.c_int32),
                ("cold_marked", ctypes.c_int32)]


class Norm(ctypes.Structure):
    _fields_ = [("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("eps", ctypes.c_double), ("scale", ctypes.c_double),
                ("flags", ctypes.c_uint32)]


class NormGradPointers(ctypes.Structure):
    _fields_ = [("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p),
                ("gate", ctypes.c_void_p)]


class GroupNorm(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("eps", ctypes.c_double), ("graphs", ctypes.c_int32), ("F", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class Grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("count", ctypes.c_int64), ("flags", ctypes.c_uint32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python paper_2609_01983_amd/build.py`")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, U32, U64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64, \
        ctypes.c_size_t
    sig = {
        "dualgcn_status_str": ([ctypes.c_int], ctypes.c_char_p),
        "dualgcn_last_hip_error": ([], ctypes.c_int),
        "dualgcn_partition": ([ctypes.POINTER(Csr), U64, U32, U32, ctypes.POINTER(Thresholds), P,
                               ctypes.POINTER(P)], ctypes.c_int),
        "dualgcn_plan_destroy": ([P], None),
        "dualgcn_spmm": ([P, P, P, I32, P], ctypes.c_int),
        "dualgcn_spmm_act": ([P, P, P, I32, U32, P], ctypes.c_int),
        "dualgcn_spmm_update": ([P, P, P, P, P, I32, I32, U32, P], ctypes.c_int),
        "dualgcn_spmm_update_route": ([P, I32, I32, P], ctypes.c_int),
        "dualgcn_update": ([P, P, P, I32, I32, I32, U32, P], ctypes.c_int),
        "dualgcn_gcn_layer_workspace": ([P, I32, I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_gcn_layer": ([P, P, P, P, I32, I32, U32, P, SZ, P], ctypes.c_int),
        "dualgcn_plan_query": ([P, ctypes.POINTER(PlanInfo)], ctypes.c_int),
        "dualgcn_plan_export": ([P, P, P, P], ctypes.c_int),
        "dualgcn_arw_patterns": ([ctypes.POINTER(Csr), U64, U32, U32, P, P], ctypes.c_int),
        "dualgcn_plan_save": ([P, P, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_plan_load": ([ctypes.POINTER(Csr), P, SZ, P, ctypes.POINTER(P)], ctypes.c_int),
        "dualgcn_aggregator_values": ([ctypes.POINTER(Csr), I32, ctypes.c_float, P, P], ctypes.c_int),
        "dualgcn_softmax_xent": ([P, P, I32, I32, ctypes.c_float, P, P, P], ctypes.c_int),
        "dualgcn_weight_grad_workspace": ([I32, I32, I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_weight_grad": ([P, P, P, I32, I32, I32, U32, ctypes.c_float, P, P, SZ, P],
                                ctypes.c_int),
        "dualgcn_weight_grad_noalloc": ([P, P, P, I32, I32, I32, U32, ctypes.c_float, P, P],
                                        ctypes.c_int),
        "dualgcn_backward_data": ([P, P, P, P, I32, I32, I32, U32, P], ctypes.c_int),
        "dualgcn_norm_residual": ([ctypes.POINTER(Norm), P, P, P, P, I32, I32, P], ctypes.c_int),
        "dualgcn_norm_residual_backward_workspace": ([I32, I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_norm_residual_backward": ([ctypes.POINTER(Norm), P, P, P, P, P, P,
                                            ctypes.POINTER(NormGradPointers), I32, I32, P, SZ, P],
                                           ctypes.c_int),
        "dualgcn_distill_workspace": ([I32, I32, I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_distill_xent": ([P, P, P, P, I32, I32, I32, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                  U32, P, P, P, SZ, P], ctypes.c_int),
        "dualgcn_quantize_fp8": ([P, I32, I32, U32, P, P, P], ctypes.c_int),
        "dualgcn_quantize_weight_fp8": ([P, I32, I32, I32, P, P, P], ctypes.c_int),
        "dualgcn_update_fp8": ([P, P, P, P, P, I32, I32, I32, U32, P], ctypes.c_int),
        "dualgcn_group_norm_act_workspace": ([ctypes.POINTER(GroupNorm), I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_group_norm_act": ([ctypes.POINTER(GroupNorm), P, P, P, I32, P, SZ, P], ctypes.c_int),
        "dualgcn_group_norm_act_backward_workspace": ([ctypes.POINTER(GroupNorm), I32, ctypes.POINTER(SZ)],
                                                      ctypes.c_int),
        "dualgcn_group_norm_act_backward": ([ctypes.POINTER(GroupNorm), P, P, P, P, P, P, I32, P, SZ, P], ctypes.c_int),
        "dualgcn_grad_norm_workspace": ([I32, ctypes.POINTER(SZ)], ctypes.c_int),
        "dualgcn_grad_norm": ([ctypes.POINTER(Grad), I32, P, P, SZ, P], ctypes.c_int),
        "dualgcn_clip_grads": ([ctypes.POINTER(Grad), I32, ctypes.c_double, ctypes.c_double, P, P, SZ, P], ctypes.c_int),
        "dualgcn_clipped_sgd": ([ctypes.POINTER(Grad), I32, ctypes.c_double, ctypes.c_double, ctypes.c_double, P, P, SZ,
                                 P], ctypes.c_int),
        "dualgcn_quantize_mxfp4": ([P, I32, I32, U32, P, P, P], ctypes.c_int),
        "dualgcn_quantize_weight_mxfp4": ([P, I32, I32, I32, P, P, P], ctypes.c_int),
        "dualgcn_dequantize_mxfp4": ([P, P, I32, I32, U32, P, P], ctypes.c_int),
        "dualgcn_update_mxfp4": ([P, P, P, P, P, I32, I32, I32, U32, P], ctypes.c_int),
        "dualgcn_bandwidth_probe": ([I32, P, P, SZ, P], ctypes.c_int),
        "dualgcn_bandwidth_probe_out_floats": ([], I32),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    return L


_lib = _load()


def lib():
    return _lib


def status_str(status):
    return _lib.dualgcn_status_str(status).decode()


def _check(status, what):
    if status != OK:
        raise DualGCNError(status, what)


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t, dtype, name):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def make_csr(rowptr, col, val):
    _dev(rowptr, torch.int32, "rowptr")
    _dev(col, torch.int32, "col")
    _dev(val, torch.float32, "val")
    n = rowptr.numel() - 1
    return Csr(n, col.numel(), rowptr.data_ptr(), col.data_ptr() if col.numel() else None,
               val.data_ptr() if val.numel() else None)


class Plan:
    """The dual-metric partition of one CSR matrix (device arrays, borrowed)."""

    def __init__(self, rowptr, col, val, seed=0, walks_per_node=16, walk_len=5,
                 alpha=(1, 2), beta=(1, 2), force_mode="auto", stream=None):
        self._keep = (rowptr, col, val)        # the plan borrows these arrays
        self.csr = make_csr(rowptr, col, val)
        self.n = self.csr.n
        th = Thresholds(alpha[0], alpha[1], beta[0], beta[1], _FORCE[force_mode])
        out = ctypes.c_void_p()
        _check(_lib.dualgcn_partition(ctypes.byref(self.csr), seed, walks_per_node, walk_len,
                                      ctypes.byref(th), _stream(stream), ctypes.byref(out)),
               "dualgcn_partition")
        self._h = out

    @property
    def handle(self):
        if not self._h:
            raise ValueError("plan destroyed")
        return self._h

    def info(self):
        pi = PlanInfo()
        _check(_lib.dualgcn_plan_query(self.handle, ctypes.byref(pi)), "dualgcn_plan_query")
        d = {name: getattr(pi, name) for name, _ in PlanInfo._fields_}
        d["s1"] = (d.pop("s1_hi") << 64) | d.pop("s1_lo")
        d["s2"] = (d.pop("s2_hi") << 64) | d.pop("s2_lo")
        return d

    def export(self):
        """(perm int32[n], S uint32[n], K uint64[n]) as numpy arrays."""
        import numpy as np
        perm = np.empty(self.n, dtype=np.int32)
        S = np.empty(self.n, dtype=np.uint32)
        K = np.empty(self.n, dtype=np.uint64)
        _check(_lib.dualgcn_plan_export(self.handle, perm.ctypes.data, S.ctypes.data,
                                        K.ctypes.data), "dualgcn_plan_export")
        return perm, S, K

    def save(self):
        """The plan as bytes (parameters, checksum of the structure, density sums)."""
        nbytes = ctypes.c_size_t()
        _check(_lib.dualgcn_plan_save(self.handle, None, ctypes.byref(nbytes)), "dualgcn_plan_save")
        buf = ctypes.create_string_buffer(nbytes.value)
        _check(_lib.dualgcn_plan_save(self.handle, buf, ctypes.byref(nbytes)), "dualgcn_plan_save")
        return buf.raw[:nbytes.value]

    @classmethod
    def load(cls, rowptr, col, val, blob, stream=None):
        """Rebuilds a saved plan on the same structure (values may differ), without walks."""
        self = cls.__new__(cls)
        self._keep = (rowptr, col, val)
        self.csr = make_csr(rowptr, col, val)
        self.n = self.csr.n
        out = ctypes.c_void_p()
        buf = ctypes.create_string_buffer(bytes(blob), len(blob))
        _check(_lib.dualgcn_plan_load(ctypes.byref(self.csr), buf, len(blob), _stream(stream),
                                      ctypes.byref(out)), "dualgcn_plan_load")
        self._h = out
        return self

    def destroy(self):
        if getattr(self, "_h", None):
            _lib.dualgcn_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def spmm(plan, X, Y=None, relu=False, out_bf16=False, stream=None):
    """Y = A X (or relu(A X)) on the plan's matrix.  X: float32 [n, F] on the device.

    With out_bf16, Y is bfloat16: the nearest-even rounding of the float32 result."""
    _dev(X, torch.float32, "X")
    if X.dim() != 2 or X.shape[0] != plan.n:
        raise ValueError("X must be [n, F]")
    ydt = torch.bfloat16 if out_bf16 else torch.float32
    if Y is None:
        Y = torch.empty(X.shape, dtype=ydt, device=X.device)
    _dev(Y, ydt, "Y")
    if Y.shape != X.shape:
        raise ValueError("Y must have X's shape")
    if relu or out_bf16:
        flags = (RELU if relu else 0) | (OUT_BF16 if out_bf16 else 0)
        _check(_lib.dualgcn_spmm_act(plan.handle, X.data_ptr(), Y.data_ptr(), X.shape[1], flags,
                                     _stream(stream)), "dualgcn_spmm_act")
    else:
        _check(_lib.dualgcn_spmm(plan.handle, X.data_ptr(), Y.data_ptr(), X.shape[1],
                                 _stream(stream)), "dualgcn_spmm")
    return Y


def update(X, W, T=None, stream=None):
    """T = X W on the bf16 matrix cores (float32 accumulation).  X: [n, F_in] float32 or
    bfloat16, W: [F_in, F_out] float32.

    Needs no plan: it may run on another stream while a partition is built."""
    if not isinstance(X, torch.Tensor) or X.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("X must be a float32 or bfloat16 tensor")
    _dev(X, X.dtype, "X")
    _dev(W, torch.float32, "W")
    F_in, F_out = W.shape
    if X.dim() != 2 or X.shape[1] != F_in:
        raise ValueError("X must be [n, F_in]")
    n = X.shape[0]
    if T is None:
        T = torch.empty((n, F_out), dtype=torch.float32, device=X.device)
    _dev(T, torch.float32, "T")
    if T.shape != (n, F_out):
        raise ValueError("T must be [n, F_out]")
    flags = IN_BF16 if X.dtype == torch.bfloat16 else 0
    _check(_lib.dualgcn_update(X.data_ptr(), W.data_ptr(), T.data_ptr(), n, F_in, F_out, flags,
                               _stream(stream)), "dualgcn_update")
    return T


def spmm_update_route(plan, F_in, F_out):
    """True when the fused kernel is the faster route of spmm_update on this plan and shape."""
    fused = ctypes.c_int32()
    _check(_lib.dualgcn_spmm_update_route(plan.handle, F_in, F_out, ctypes.byref(fused)),
           "dualgcn_spmm_update_route")
    return bool(fused.value)


def spmm_update(plan, X, W, T=None, relu=False, H=None, stream=None):
    """T = bf16(act(A X)) bf16(W) (float32 accumulation): the aggregation of one layer fused
    with the next layer's update.  X: float32 [n, F_in], W: float32 [F_in, F_out],
    T: float32 [n, F_out].  H: None (act(A X) is not kept), or a bfloat16 [n, F_in]
    tensor that receives bf16(act(A X)).  Where the library's two-call route is the faster
    one and no H is given, a temporary H is allocated for it (the same T either way)."""
    _dev(X, torch.float32, "X")
    _dev(W, torch.float32, "W")
    if X.dim() != 2 or X.shape[0] != plan.n:
        raise ValueError("X must be [n, F_in]")
    F_in, F_out = W.shape
    if X.shape[1] != F_in:
        raise ValueError("W must be [F_in, F_out]")
    if T is None:
        T = torch.empty((plan.n, F_out), dtype=torch.float32, device=X.device)
    _dev(T, torch.float32, "T")
    if T.shape != (plan.n, F_out):
        raise ValueError("T must be [n, F_out]")
    hp = None
    if H is not None:
        _dev(H, torch.bfloat16, "H")
        if H.shape != (plan.n, F_in):
            raise ValueError("H must be [n, F_in]")
        hp = H.data_ptr()
    elif not spmm_update_route(plan, F_in, F_out):
        hp = torch.empty((plan.n, F_in), dtype=torch.bfloat16, device=X.device).data_ptr()
    _check(_lib.dualgcn_spmm_update(plan.handle, X.data_ptr(), W.data_ptr(), T.data_ptr(), hp,
                                    F_in, F_out, RELU if relu else 0, _stream(stream)),
           "dualgcn_spmm_update")
    return T


def gcn_layer_workspace_bytes(plan, F_in, F_out):
    nbytes = ctypes.c_size_t()
    _check(_lib.dualgcn_gcn_layer_workspace(plan.handle, F_in, F_out, ctypes.byref(nbytes)),
           "dualgcn_gcn_layer_workspace")
    return nbytes.value


def gcn_layer(plan, X, W, relu=False, Y=None, workspace=None, out_bf16=False, stream=None):
    """Y = act(A (X W)) with X W on the bf16 matrix cores (float32 accumulation).

    X may be float32 or bfloat16; with out_bf16 Y is the bfloat16 rounding of the result."""
    if not isinstance(X, torch.Tensor) or X.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("X must be a float32 or bfloat16 tensor")
    _dev(X, X.dtype, "X")
    _dev(W, torch.float32, "W")
    F_in, F_out = W.shape
    if X.shape != (plan.n, F_in):
        raise ValueError("X must be [n, F_in]")
    ydt = torch.bfloat16 if out_bf16 else torch.float32
    if Y is None:
        Y = torch.empty((plan.n, F_out), dtype=ydt, device=X.device)
    _dev(Y, ydt, "Y")
    need = gcn_layer_workspace_bytes(plan, F_in, F_out)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    _dev(workspace, torch.uint8, "workspace")
    flags = (RELU if relu else 0) | (IN_BF16 if X.dtype == torch.bfloat16 else 0) | \
        (OUT_BF16 if out_bf16 else 0)
    _check(_lib.dualgcn_gcn_layer(plan.handle, X.data_ptr(), W.data_ptr(), Y.data_ptr(), F_in,
                                  F_out, flags, workspace.data_ptr(),
                                  workspace.numel(), _stream(stream)), "dualgcn_gcn_layer")
    return Y


# ------------------------------------------------------------------ aggregators

AGG_GCN, AGG_MEAN, AGG_SUM = 0, 1, 2
_AGG = {"gcn": AGG_GCN, "mean": AGG_MEAN, "sum": AGG_SUM,
        AGG_GCN: AGG_GCN, AGG_MEAN: AGG_MEAN, AGG_SUM: AGG_SUM}


def aggregator_values(rowptr, col, kind="gcn", eps=0.0, val=None, stream=None):
    """float32 values of an aggregation matrix on this structure: "gcn" 1/sqrt(d_r d_c),
    "mean" 1/d_r, "sum" 1 with 1 + eps on self-loops (GIN).  Validates the CSR (waits)."""
    if val is None:
        val = torch.empty(col.numel(), dtype=torch.float32, device=col.device)
    csr = make_csr(rowptr, col, val)
    _check(_lib.dualgcn_aggregator_values(ctypes.byref(csr), _AGG[kind], float(eps),
                                          val.data_ptr() if val.numel() else None,
                                          _stream(stream)), "dualgcn_aggregator_values")
    return val


# ------------------------------------------------------------------ training

def _float_or_bf16(t, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{name} must be a float32 or bfloat16 tensor")
    _dev(t, t.dtype, name)
    if t.dim() != 2:
        raise ValueError(f"{name} must be 2-D")


def softmax_xent(Y, labels, scale=None, G=None, loss=None, stream=None):
    """Softmax cross-entropy over the rows whose label is in [0, C).

    Returns (G, loss): G = dloss/dY (float32 [n, C]) and a float64 device tensor of
    LOSS_SLOTS entries whose entry 0 is the loss.  scale defaults to 1 / (labeled rows),
    counted on the host from `labels` only when not given."""
    _dev(Y, torch.float32, "Y")
    _dev(labels, torch.int32, "labels")
    n, C = Y.shape
    if labels.shape != (n,):
        raise ValueError("labels must be [n]")
    if scale is None:
        scale = 1.0 / max(1, int(((labels >= 0) & (labels < C)).sum().item()))
    if G is None:
        G = torch.empty_like(Y)
    _dev(G, torch.float32, "G")
    if loss is None:
        loss = torch.empty(LOSS_SLOTS, dtype=torch.float64, device=Y.device)
    _dev(loss, torch.float64, "loss")
    if G.shape != Y.shape or loss.numel() < LOSS_SLOTS:
        raise ValueError("G must match Y and loss must hold LOSS_SLOTS entries")
    _check(_lib.dualgcn_softmax_xent(Y.data_ptr(), labels.data_ptr(), n, C, float(scale),
                                     G.data_ptr(), loss.data_ptr(), _stream(stream)),
           "dualgcn_softmax_xent")
    return G, loss


def weight_grad_workspace_bytes(n, F_in, F_out):
    nbytes = ctypes.c_size_t()
    _check(_lib.dualgcn_weight_grad_workspace(n, F_in, F_out, ctypes.byref(nbytes)),
           "dualgcn_weight_grad_workspace")
    return nbytes.value


def weight_grad(X, G, dW=None, lr=0.0, W=None, workspace=None, stream=None):
    """dW = X^T G on the bf16 matrix cores; with W, also the SGD step W -= lr dW.
    X: [n, F_in] and G: [n, F_out], each float32 or bfloat16."""
    _float_or_bf16(X, "X")
    _float_or_bf16(G, "G")
    n, F_in = X.shape
    if G.shape[0] != n:
        raise ValueError("X and G must have the same rows")
    F_out = G.shape[1]
    if dW is None:
        dW = torch.empty((F_in, F_out), dtype=torch.float32, device=X.device)
    _dev(dW, torch.float32, "dW")
    if W is not None:
        _dev(W, torch.float32, "W")
        if W.shape != (F_in, F_out):
            raise ValueError("W must be [F_in, F_out]")
    if dW.shape != (F_in, F_out):
        raise ValueError("dW must be [F_in, F_out]")
    need = weight_grad_workspace_bytes(n, F_in, F_out)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    flags = (IN_BF16 if X.dtype == torch.bfloat16 else 0) | \
            (GRAD_BF16 if G.dtype == torch.bfloat16 else 0)
    _check(_lib.dualgcn_weight_grad(X.data_ptr(), G.data_ptr(), dW.data_ptr(), n, F_in, F_out,
                                    flags, float(lr), W.data_ptr() if W is not None else None,
                                    workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                    _stream(stream)), "dualgcn_weight_grad")
    return dW


def weight_grad_noalloc(X, G, dW, lr=0.0, W=None, stream=None):
    """dualgcn_weight_grad_noalloc: weight_grad with the partial products in the library's
    static device array (no workspace, nothing allocated by the library).  dW [F_in, F_out]
    float32 is the caller's."""
    _float_or_bf16(X, "X")
    _float_or_bf16(G, "G")
    n, F_in = X.shape
    if G.shape[0] != n:
        raise ValueError("X and G must have the same rows")
    F_out = G.shape[1]
    _dev(dW, torch.float32, "dW")
    if dW.shape != (F_in, F_out):
        raise ValueError("dW must be [F_in, F_out]")
    if W is not None:
        _dev(W, torch.float32, "W")
        if W.shape != (F_in, F_out):
            raise ValueError("W must be [F_in, F_out]")
    flags = (IN_BF16 if X.dtype == torch.bfloat16 else 0) | \
            (GRAD_BF16 if G.dtype == torch.bfloat16 else 0)
    _check(_lib.dualgcn_weight_grad_noalloc(X.data_ptr(), G.data_ptr(), dW.data_ptr(), n, F_in,
                                            F_out, flags, float(lr),
                                            W.data_ptr() if W is not None else None,
                                            _stream(stream)), "dualgcn_weight_grad_noalloc")
    return dW


def backward_data(G, W, M=None, dX=None, stream=None):
    """dX = (G W^T) * [M > 0] on the bf16 matrix cores (no mask without M).
    G: [n, F_out] float32 or bfloat16, W: [F_in, F_out] float32, M: [n, F_in]."""
    _float_or_bf16(G, "G")
    _dev(W, torch.float32, "W")
    F_in, F_out = W.shape
    n = G.shape[0]
    if G.shape[1] != F_out:
        raise ValueError("G must be [n, F_out]")
    flags = GRAD_BF16 if G.dtype == torch.bfloat16 else 0
    if M is not None:
        _float_or_bf16(M, "M")
        if M.shape != (n, F_in):
            raise ValueError("M must be [n, F_in]")
        flags |= IN_BF16 if M.dtype == torch.bfloat16 else 0
    if dX is None:
        dX = torch.empty((n, F_in), dtype=torch.float32, device=G.device)
    _dev(dX, torch.float32, "dX")
    if dX.shape != (n, F_in):
        raise ValueError("dX must be [n, F_in]")
    _check(_lib.dualgcn_backward_data(G.data_ptr(), W.data_ptr(),
                                      M.data_ptr() if M is not None else None, dX.data_ptr(), n,
                                      F_in, F_out, flags, _stream(stream)), "dualgcn_backward_data")
    return dX


# ------------------------------------------------------------------ deep GCNs

# A call's host time counts where the work is small, so its checks take the plain attribute tests
# first (several microseconds less than building stream and device objects).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _queue(stream, *tensors):
    """The HIP stream a call goes to.  Every tensor, and the stream, is on the current device: the
    library launches there."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"tensor on {t.device}, the current device is cuda:{device}")
    if stream is None:
        return _raw_stream(device)
    if stream.device.index != device:
        raise ValueError(f"stream on {stream.device}, the current device is cuda:{device}")
    return stream.cuda_stream


def _empty(shape, dtype, like, stream):
    """Device memory for work queued on `stream`: taken from that stream's pool, so that it is
    neither still in use by an earlier owner nor handed on while the work runs."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _shaped(t, dtype, shape, name):
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous()):
        _dev(t, dtype, name)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return t


def _rows(t, name):
    """A float32 or bfloat16 matrix: is it bfloat16?"""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.is_contiguous() and
            (t.dtype is torch.float32 or t.dtype is torch.bfloat16)):
        _float_or_bf16(t, name)
    if t.shape[0] > 0x7FFFFFFF or t.shape[1] > 0x7FFFFFFF:
        raise ValueError(f"{name} has more than 2^31 - 1 rows or columns")
    return t.dtype is torch.bfloat16


def _norm(R, B, post_norm, post_weight, post_bias, gate, gate_sigmoid, scale, pre_weight, pre_bias, kind, eps):
    """The checked parameters of a block's norms, as the library takes them."""
    if kind != "rms" and kind != "layer":
        raise ValueError('kind must be "rms" or "layer"')
    n, F = R.shape
    flags = NORM_LAYER if kind == "layer" else 0
    if post_norm:
        flags |= NORM_POST
    if _rows(R, "R"):
        flags |= STREAM_BF16
    width = (F,)
    if post_weight is not None:
        _shaped(post_weight, torch.float32, width, "post_weight")
    if post_bias is not None:
        _shaped(post_bias, torch.float32, width, "post_bias")
    if pre_weight is not None:
        _shaped(pre_weight, torch.float32, width, "pre_weight")
    if pre_bias is not None:
        _shaped(pre_bias, torch.float32, width, "pre_bias")
    if B is not None:
        if _rows(B, "B"):
            flags |= IN_BF16
        _shaped(B, B.dtype, (n, F), "B")
    if gate is not None:
        if B is None:
            raise ValueError("a gate needs a block B")
        if gate.dim() == 1:
            _shaped(gate, torch.float32, width, "gate")
            flags |= GATE_FEATURE
        elif gate.dim() == 2 and gate.shape[1] == 1 and (F != 1 or gate.dtype is not B.dtype):
            _shaped(gate, torch.float32, (n, 1), "gate")
            flags |= GATE_NODE
        else:
            _shaped(gate, B.dtype, (n, F), "gate")
            flags |= GATE_FULL
    if gate_sigmoid:
        flags |= GATE_SIGMOID
    return Norm(_ptr(post_weight), _ptr(post_bias), _ptr(pre_weight), _ptr(pre_bias), _ptr(gate), eps, scale, flags)


def norm_residual(R, B=None, *, post_norm=True, post_weight=None, post_bias=None, gate=None,
                  gate_sigmoid=False, scale=1.0, pre_norm=True, pre_weight=None, pre_bias=None,
                  kind="rms", eps=1e-5, norm_bf16=False, Rn=None, Z=None, stream=None):
    """What stands between two residual blocks: Rn = R + scale * gate * post(B), Z = pre(Rn).

    R: [n, F] float32 or bfloat16 (the residual stream); B: [n, F] float32 or bfloat16 (the
    block's output), or None before the first block (Rn is then R itself, and Z = pre(R)).
    post and pre are RMS norms (kind "rms") or layer norms ("layer") with float32 [F] weights and
    biases (None: ones and zeros); post_norm=False leaves the block as it is, pre_norm=False
    makes no Z.  gate: None, float32 [F] (one for each feature), float32 [n, 1] (one for each
    node), or [n, F] in B's type; with gate_sigmoid it holds logits.  Z is float32, or bfloat16
    with norm_bf16 (what `update` takes).  Z norms Rn as it is stored; a bfloat16 Rn beside a float32 Z
    is summed in float64, rounded to float32 and stored.  Rn may be R (in place).  Returns (Rn, Z)."""
    _rows(R, "R")
    n, F = shape = R.shape
    if B is None:
        if not pre_norm:
            raise ValueError("nothing to do: no block and no norm")
        if Rn is not None and Rn is not R:
            raise ValueError("Rn is R where there is no block")
        post_norm = False
    p = _norm(R, B, post_norm, post_weight, post_bias, gate, gate_sigmoid, scale, pre_weight, pre_bias, kind, eps)
    s = _queue(stream, R, B, post_weight, post_bias, gate, pre_weight, pre_bias, Rn, Z)
    if B is not None:
        Rn = _empty(shape, R.dtype, R, stream) if Rn is None else _shaped(Rn, R.dtype, shape, "Rn")
    if pre_norm:
        zdt = torch.bfloat16 if norm_bf16 else torch.float32
        Z = _empty(shape, zdt, R, stream) if Z is None else _shaped(Z, zdt, shape, "Z")
        if norm_bf16:
            p.flags |= OUT_BF16
    elif Z is not None:
        raise ValueError("Z without pre_norm")
    _check(_lib.dualgcn_norm_residual(p, R.data_ptr(), _ptr(B), None if B is None else Rn.data_ptr(), _ptr(Z), n, F, s),
           "dualgcn_norm_residual")
    return (R if B is None else Rn), Z


class NormGrads(collections.namedtuple("NormGrads", "R B gate post_weight post_bias pre_weight pre_bias")):
    """Gradients of norm_residual's operands; None where there is no such operand."""
    __slots__ = ()


def norm_residual_backward_workspace_bytes(n, F):
    nbytes = ctypes.c_size_t()
    _check(_lib.dualgcn_norm_residual_backward_workspace(n, F, ctypes.byref(nbytes)),
           "dualgcn_norm_residual_backward_workspace")
    return nbytes.value


def norm_residual_backward(Rn, B=None, dZ=None, dRn=None, *, post_norm=True, post_weight=None, post_bias=None,
                           gate=None, gate_sigmoid=False, scale=1.0, pre_norm=True, pre_weight=None,
                           pre_bias=None, kind="rms", eps=1e-5, grad_bf16=False, dR=None, dB=None,
                           workspace=None, stream=None):
    """Gradients of norm_residual: Rn is the stream it returned, B and the parameters are its own.

    dZ: gradient of Z (None: none), float32, or bfloat16 with grad_bf16; dRn: gradient of Rn from
    elsewhere, in Rn's type (None: zeros); not both None.  Returns NormGrads: R in Rn's type (dR
    may be dRn), B and a full gate in dZ's type, the vectors in float32 ([F], or [n, 1] for a
    gate per node).  A weight or bias that is None has no gradient."""
    _rows(Rn, "Rn")
    n, F = shape = Rn.shape
    if B is None:
        post_norm = False
        if dB is not None:
            raise ValueError("dB without B")
    if not pre_norm and dZ is not None:
        raise ValueError("dZ without pre_norm")
    p = _norm(Rn, B, post_norm, post_weight, post_bias, gate, gate_sigmoid, scale, pre_weight, pre_bias, kind, eps)
    gdt = torch.float32
    if grad_bf16:
        gdt = torch.bfloat16
        p.flags |= GRAD_BF16
    s = _queue(stream, Rn, B, dZ, dRn, post_weight, post_bias, gate, pre_weight, pre_bias, dR, dB, workspace)
    if dZ is not None:
        _shaped(dZ, gdt, shape, "dZ")
    if dRn is not None:
        _shaped(dRn, Rn.dtype, shape, "dRn")
    dR = _empty(shape, Rn.dtype, Rn, stream) if dR is None else _shaped(dR, Rn.dtype, shape, "dR")
    if B is not None:
        dB = _empty(shape, gdt, Rn, stream) if dB is None else _shaped(dB, gdt, shape, "dB")
    dgate = None
    if gate is not None:
        dgate = _empty(gate.shape, gdt if p.flags & GATE_FULL else torch.float32, Rn, stream)
    # the vectors' gradients: one piece of memory, a row each
    want = [post_weight is not None, post_bias is not None, pre_weight is not None and dZ is not None,
            pre_bias is not None and dZ is not None]
    rows = iter(_empty((sum(want), F), torch.float32, Rn, stream).unbind(0) if any(want) else ())
    vec = [next(rows) if w else None for w in want]
    out = NormGrads(dR, dB, dgate, *vec)
    if workspace is None:
        workspace = _empty((norm_residual_backward_workspace_bytes(n, F),), torch.uint8, Rn, stream)
    else:
        _dev(workspace, torch.uint8, "workspace")
    g = NormGradPointers(_ptr(vec[0]), _ptr(vec[1]), _ptr(vec[2]), _ptr(vec[3]), _ptr(dgate))
    _check(_lib.dualgcn_norm_residual_backward(p, Rn.data_ptr(), _ptr(B), _ptr(dZ), _ptr(dRn), dR.data_ptr(), _ptr(dB),
                                               g, n, F, workspace.data_ptr(), workspace.numel(), s),
           "dualgcn_norm_residual_backward")
    return out


def distill_workspace_bytes(n, C, K):
    nbytes = ctypes.c_size_t()
    _check(_lib.dualgcn_distill_workspace(n, C, K, ctypes.byref(nbytes)), "dualgcn_distill_workspace")
    return nbytes.value


def distill_xent(Y, ids, teacher, labels=None, temperature=1.0, soft_scale=None, hard_scale=None,
                 grad_bf16=False, G=None, loss=None, workspace=None, stream=None):
    """The loss of a student's logits Y against its teacher's top logits, and its gradient.

    Y: [n, C] float32 or bfloat16; ids: int32 [n, K] classes kept of each row's teacher, teacher:
    [n, K] float32 or bfloat16 their logits (an id outside [0, C) or a logit of -inf: no entry);
    labels: int32 [n] or None.  Returns (G, loss): G = dloss[0]/dY ([n, C] float32, or bfloat16
    with grad_bf16) and the float32 device tensor loss = [soft + hard, soft, hard], soft =
    soft_scale T^2 sum KL(teacher || softmax(Y / T)), hard = hard_scale sum of the labels'
    cross-entropy.  Past a temperature of 8 soft is formed in float64, by a second pass over Y.
    The scales default to 1 / (rows with an entry) and 1 / (labeled rows), counted on the host only
    when not given."""
    flags = IN_BF16 if _rows(Y, "Y") else 0
    n, C = shape = Y.shape
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be an [n, K] tensor")
    K = ids.shape[1]
    if max(C, K) > 0x7FFFFFFF:
        raise ValueError("more than 2^31 - 1 classes or entries")
    _shaped(ids, torch.int32, (n, K), "ids")
    if _rows(teacher, "teacher"):
        flags |= TEACHER_BF16
    _shaped(teacher, teacher.dtype, (n, K), "teacher")
    if labels is not None:
        _shaped(labels, torch.int32, (n,), "labels")
    s = _queue(stream, Y, ids, teacher, labels, G, loss, workspace)
    if hard_scale is None and labels is None:
        hard_scale = 0.0
    if soft_scale is None or hard_scale is None:
        with torch.cuda.stream(stream):              # the operands are ready on the call's stream
            if soft_scale is None:
                kept = (ids >= 0) & (ids < C) & (teacher != float("-inf"))
                soft_scale = 1.0 / max(1, int(kept.any(1).sum().item()))
            if hard_scale is None:
                hard_scale = 1.0 / max(1, int(((labels >= 0) & (labels < C)).sum().item()))
    gdt = torch.float32
    if grad_bf16:
        gdt = torch.bfloat16
        flags |= GRAD_BF16
    G = _empty(shape, gdt, Y, stream) if G is None else _shaped(G, gdt, shape, "G")
    loss = _empty((3,), torch.float32, Y, stream) if loss is None else _shaped(loss, torch.float32, (3,), "loss")
    if workspace is None:
        workspace = _empty((distill_workspace_bytes(n, C, K),), torch.uint8, Y, stream)
    else:
        _dev(workspace, torch.uint8, "workspace")
    _check(_lib.dualgcn_distill_xent(Y.data_ptr(), ids.data_ptr(), teacher.data_ptr(), _ptr(labels), n, C, K,
                                     temperature, soft_scale, hard_scale, flags, G.data_ptr(), loss.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), s), "dualgcn_distill_xent")
    return G, loss


def _fp8_blocks(F):
    return (F + FP8_BLOCK - 1) // FP8_BLOCK


def _fp8_out(like, shape, blocks, Q, scales, stream):
    e4m3 = torch.float8_e4m3fn
    Q = _empty(shape, e4m3, like, stream) if Q is None else _shaped(Q, e4m3, shape, "Q")
    if scales is None:
        return Q, _empty(blocks, torch.float32, like, stream)
    return Q, _shaped(scales, torch.float32, blocks, "scales")


def quantize_fp8(X, Q=None, scales=None, stream=None):
    """(Q, scales): X ([n, F] float32 or bfloat16) as float8_e4m3fn [n, F] with a float32 scale, a
    power of two, for each 128 consecutive features of a row ([n, ceil(F / 128)])."""
    flags = IN_BF16 if _rows(X, "X") else 0
    n, F = X.shape
    s = _queue(stream, X, Q, scales)
    Q, scales = _fp8_out(X, (n, F), (n, _fp8_blocks(F)), Q, scales, stream)
    _check(_lib.dualgcn_quantize_fp8(X.data_ptr(), n, F, flags, Q.data_ptr(), scales.data_ptr(), s),
           "dualgcn_quantize_fp8")
    return Q, scales


def quantize_weight_fp8(W, transpose=True, Q=None, scales=None, stream=None):
    """(Q, scales): W ([F_in, F_out] float32) as float8_e4m3fn with a float32 scale for each 128 x 128
    block, as update_fp8 reads it: [F_out, F_in] for X W, or with transpose=False [F_in, F_out]
    for the gradient's product G W^T."""
    _dev(W, torch.float32, "W")
    if W.dim() != 2:
        raise ValueError("W must be [F_in, F_out]")
    F_in, F_out = W.shape
    if max(F_in, F_out) > 0x7FFFFFFF:
        raise ValueError("more than 2^31 - 1 rows or columns")
    s = _queue(stream, W, Q, scales)
    shape = (F_out, F_in) if transpose else (F_in, F_out)
    Q, scales = _fp8_out(W, shape, (_fp8_blocks(shape[0]), _fp8_blocks(shape[1])), Q, scales, stream)
    _check(_lib.dualgcn_quantize_weight_fp8(W.data_ptr(), F_in, F_out, 1 if transpose else 0, Q.data_ptr(),
                                            scales.data_ptr(), s), "dualgcn_quantize_weight_fp8")
    return Q, scales


def update_fp8(X, sx, W, sw, T=None, out_bf16=False, stream=None):
    """T = X W from 8-bit operands on the matrix cores: X float8_e4m3fn [n, F_in] with its float32
    scales sx [n, ceil(F_in / 128)], W float8_e4m3fn [F_out, F_in] (transposed) with sw
    [ceil(F_out / 128), ceil(F_in / 128)].  T is float32 [n, F_out], or bfloat16 with out_bf16."""
    if not (isinstance(X, torch.Tensor) and isinstance(W, torch.Tensor)) or X.dim() != 2 or W.dim() != 2:
        raise ValueError("X must be an [n, F_in] tensor and W an [F_out, F_in] tensor")
    n, F_in = X.shape
    F_out = W.shape[0]
    if max(n, F_in, F_out) > 0x7FFFFFFF:
        raise ValueError("more than 2^31 - 1 rows or columns")
    _shaped(X, torch.float8_e4m3fn, (n, F_in), "X")
    _shaped(W, torch.float8_e4m3fn, (F_out, F_in), "W")
    _shaped(sx, torch.float32, (n, _fp8_blocks(F_in)), "sx")
    _shaped(sw, torch.float32, (_fp8_blocks(F_out), _fp8_blocks(F_in)), "sw")
    s = _queue(stream, X, sx, W, sw, T)
    tdt = torch.bfloat16 if out_bf16 else torch.float32
    T = _empty((n, F_out), tdt, X, stream) if T is None else _shaped(T, tdt, (n, F_out), "T")
    _check(_lib.dualgcn_update_fp8(X.data_ptr(), sx.data_ptr(), W.data_ptr(), sw.data_ptr(), T.data_ptr(), n, F_in,
                                   F_out, OUT_BF16 if out_bf16 else 0, s), "dualgcn_update_fp8")
    return T


# ------------------------------------------------------------------ batches of graphs

_ACTS = {None: 0, "relu": RELU, "silu": SILU}


def _group(X, ptr, groups, weight, bias, act, eps):
    """The checked parameters of a group norm, as the library takes them."""
    flags = IN_BF16 if _rows(X, "X") else 0
    if act not in _ACTS:
        raise ValueError('act must be None, "relu" or "silu"')
    F = X.shape[1]
    if groups < 1 or F % groups:
        raise ValueError(f"groups must divide the {F} features, got {groups}")
    width = (F,)
    if weight is not None:
        _shaped(weight, torch.float32, width, "weight")
    if bias is not None:
        _shaped(bias, torch.float32, width, "bias")
    graphs = 1
    if ptr is not None:
        if not isinstance(ptr, torch.Tensor) or ptr.dim() != 1 or ptr.numel() < 2:
            raise ValueError("ptr must be an int32 tensor of one offset more than there are graphs")
        graphs = ptr.numel() - 1
        if graphs > 0x7FFFFFFF:
            raise ValueError("more than 2^31 - 1 graphs")
        _shaped(ptr, torch.int32, (graphs + 1,), "ptr")
    return GroupNorm(_ptr(ptr), _ptr(weight), _ptr(bias), eps, graphs, F, groups, flags | _ACTS[act])


def _workspace(query, what, p, n, like, workspace, stream):
    if workspace is not None:
        return _dev(workspace, torch.uint8, "workspace")
    nbytes = ctypes.c_size_t()
    _check(query(p, n, ctypes.byref(nbytes)), what)
    if nbytes.value == 0:
        return None
    return _empty((nbytes.value,), torch.uint8, like, stream)


def group_norm_workspace_bytes(n, F, groups, graphs=1, backward=False):
    """Bytes of the workspace of group_norm (or of its backward pass) for n rows of F features in `graphs` graphs."""
    p = GroupNorm(1 << 30, None, None, 1e-5, graphs, F, groups, 0)
    nbytes = ctypes.c_size_t()
    name = "dualgcn_group_norm_act_backward_workspace" if backward else "dualgcn_group_norm_act_workspace"
    _check(getattr(_lib, name)(p, n, ctypes.byref(nbytes)), name)
    return nbytes.value


def group_norm(X, ptr=None, *, groups, weight=None, bias=None, act=None, eps=1e-5, out_bf16=False, Y=None, stats=None,
               workspace=None, stream=None):
    """(Y, stats): a group norm with an activation over the nodes of each graph of a batch.

    X: [n, F] float32 or bfloat16, a row for each node; ptr: int32 [graphs + 1] on the device, graph b has the rows
    ptr[b] .. ptr[b + 1] - 1 (None: all rows are one graph).  The mean and variance go over a graph's nodes and the F / groups
    features of a group; weight and bias: float32 [F] or None; act: None, "relu" or "silu".  Y is [n, F]
    float32, or bfloat16 with out_bf16; it may be X (in place) if the types are the same.  Rows of no graph (padding) are 0 in
    a Y made here, and left as they were in one that is given.  stats: float64 [graphs, groups, 2], the mean and
    1 / sqrt(variance + eps), which group_norm_backward takes."""
    p = _group(X, ptr, groups, weight, bias, act, eps)
    n, F = shape = X.shape
    s = _queue(stream, X, ptr, weight, bias, Y, stats, workspace)
    ydt = torch.float32
    if out_bf16:
        ydt = torch.bfloat16
        p.flags |= OUT_BF16
    if Y is None:
        Y = _empty(shape, ydt, X, stream)
        p.flags |= ZERO_REST
    else:
        _shaped(Y, ydt, shape, "Y")
    if stats is None:
        stats = _empty((p.graphs, groups, 2), torch.float64, X, stream)
    else:
        _shaped(stats, torch.float64, (p.graphs, groups, 2), "stats")
    workspace = _workspace(_lib.dualgcn_group_norm_act_workspace, "dualgcn_group_norm_act_workspace", p, n, X, workspace,
                           stream)
    _check(_lib.dualgcn_group_norm_act(p, X.data_ptr(), Y.data_ptr(), stats.data_ptr(), n, _ptr(workspace),
                                       0 if workspace is None else workspace.numel(), s), "dualgcn_group_norm_act")
    return Y, stats


class GroupNormGrads(collections.namedtuple("GroupNormGrads", "X weight bias")):
    """Gradients of group_norm's operands; None where there is no such operand."""
    __slots__ = ()


def group_norm_backward(X, dY, stats, ptr=None, *, groups, weight=None, bias=None, act=None, dX=None, workspace=None,
                        stream=None):
    """GroupNormGrads of group_norm: X, ptr and the parameters are its own, stats what it returned, dY ([n, F] float32
    or bfloat16) the gradient of Y.  The gradient of X is in dY's type (dX may be dY; rows of no graph as for Y), those of
    the vectors float32 [F], None for a vector that is None."""
    p = _group(X, ptr, groups, weight, bias, act, 1e-5)
    n, F = shape = X.shape
    if _rows(dY, "dY"):
        p.flags |= GRAD_BF16
    _shaped(dY, dY.dtype, shape, "dY")
    _shaped(stats, torch.float64, (p.graphs, groups, 2), "stats")
    s = _queue(stream, X, dY, stats, ptr, weight, bias, dX, workspace)
    if dX is None:
        dX = _empty(shape, dY.dtype, X, stream)
        p.flags |= ZERO_REST
    else:
        _shaped(dX, dY.dtype, shape, "dX")
    dw = None if weight is None else _empty((F,), torch.float32, X, stream)
    db = None if bias is None else _empty((F,), torch.float32, X, stream)
    workspace = _workspace(_lib.dualgcn_group_norm_act_backward_workspace, "dualgcn_group_norm_act_backward_workspace", p,
                           n, X, workspace, stream)
    _check(_lib.dualgcn_group_norm_act_backward(p, X.data_ptr(), dY.data_ptr(), stats.data_ptr(), dX.data_ptr(), _ptr(dw),
                                                _ptr(db), n, workspace.data_ptr(), workspace.numel(), s),
           "dualgcn_group_norm_act_backward")
    return GroupNormGrads(dX, dw, db)


# ------------------------------------------------------------------ clipped gradients

def grad_norm_workspace_bytes(tensors):
    nbytes = ctypes.c_size_t()
    _check(_lib.dualgcn_grad_norm_workspace(tensors, ctypes.byref(nbytes)), "dualgcn_grad_norm_workspace")
    return nbytes.value


def _addresses(tensors, like, dtypes, name, device):
    """Where the tensors are, each of them in its dtype and in the shape of its tensor of `like`."""
    if len(tensors) != len(like):
        raise ValueError(f"as many tensors as gradients: {name}")
    at = []
    for t, g, dtype in zip(tensors, like, dtypes):
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_contiguous() and t.get_device() == device and t.shape == g.shape):
            _shaped(t, dtype, g.shape, name)
            _queue(None, t)
        at.append(t.data_ptr())
    return at


def _grads(grads, weights, out, norm, workspace, stream):
    """The list of a call on many gradients as the library takes it, and what the call needs beside it."""
    if not grads:
        raise ValueError("no gradients")
    device, f32, bf16 = torch.cuda.current_device(), torch.float32, torch.bfloat16
    at, counts, dtypes = [], [], []
    for g in grads:
        if not (isinstance(g, torch.Tensor) and ((dtype := g.dtype) is f32 or dtype is bf16) and g.is_contiguous() and g.get_device() == device):
            if not isinstance(g, torch.Tensor) or g.dtype not in (f32, bf16):
                raise TypeError("a gradient must be a float32 or bfloat16 tensor")
            _dev(g, g.dtype, "a gradient")
            _queue(None, g)
        at.append(g.data_ptr())
        counts.append(g.numel())
        dtypes.append(dtype)
    s = _queue(stream, norm, workspace)
    single, none = [f32] * len(at), [0] * len(at)
    of_weights = none if weights is None else _addresses(weights, grads, single, "a weight", device)
    if out is None:
        of_out = none
    elif weights is None and out is grads:
        of_out = at
    elif weights is not None and out is weights:
        of_out = of_weights
    else:
        of_out = _addresses(out, grads, dtypes if weights is None else single, "an output", device)
    # a Grad is five words
    words = array.array("Q", [v for row in zip(at, of_weights, of_out, counts, none) for v in row])
    for i, dtype in enumerate(dtypes):
        if dtype is bf16:
            words[5 * i + 4] = GRAD_BF16
    rows = (Grad * len(at)).from_buffer(words)
    norm = _empty((1,), f32, grads[0], stream) if norm is None else _shaped(norm, f32, (1,), "norm")
    if workspace is None:
        workspace = _empty((grad_norm_workspace_bytes(len(at)),), torch.uint8, grads[0], stream)
    else:
        _dev(workspace, torch.uint8, "workspace")
    return rows, norm, workspace, s


def grad_norm(grads, norm=None, workspace=None, stream=None):
    """The norm of all gradients together (a list of float32 and bfloat16 tensors of any shapes), float32 [1]."""
    rows, norm, workspace, s = _grads(grads, None, None, norm, workspace, stream)
    _check(_lib.dualgcn_grad_norm(rows, len(rows), norm.data_ptr(), workspace.data_ptr(), workspace.numel(), s),
           "dualgcn_grad_norm")
    return norm


def clip_grads(grads, max_norm, out=None, eps=1e-6, norm=None, workspace=None, stream=None):
    """(out, norm): the gradients scaled by min(1, max_norm / (norm + eps)), norm that of all of them together (float32
    [1], on the device: nothing is waited for).  out: tensors like the gradients; None or `grads` itself: in place."""
    if out is None:
        out = grads
    rows, norm, workspace, s = _grads(grads, None, out, norm, workspace, stream)
    _check(_lib.dualgcn_clip_grads(rows, len(rows), max_norm, eps, norm.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                   s), "dualgcn_clip_grads")
    return out, norm


def clipped_sgd(weights, grads, lr, max_norm, out=None, eps=1e-6, norm=None, workspace=None, stream=None):
    """(out, norm): weights - lr * clipped gradients (as clip_grads has them), float32; the gradients stay as they are.
    out: tensors like the weights; None or `weights` itself: in place."""
    if out is None:
        out = weights
    rows, norm, workspace, s = _grads(grads, weights, out, norm, workspace, stream)
    _check(_lib.dualgcn_clipped_sgd(rows, len(rows), max_norm, eps, lr, norm.data_ptr(), workspace.data_ptr(),
                                    workspace.numel(), s), "dualgcn_clipped_sgd")
    return out, norm


# ------------------------------------------------------------------ 4-bit operands

def _mx_blocks(F):
    return (F + MX_BLOCK - 1) // MX_BLOCK


def _mx_out(like, n, F, Q, scales, stream):
    b = _mx_blocks(F)
    Q = _empty((n, 16 * b), torch.uint8, like, stream) if Q is None else _shaped(Q, torch.uint8, (n, 16 * b), "Q")
    if scales is None:
        return Q, _empty((n, b), torch.uint8, like, stream)
    return Q, _shaped(scales, torch.uint8, (n, b), "scales")


def _mx(Q, scales, name, its):
    """A matrix in 4 bits: its rows and blocks."""
    if not isinstance(Q, torch.Tensor) or Q.dim() != 2 or Q.shape[1] % 16:
        raise ValueError(f"{name} must be a uint8 tensor [rows, 16 * blocks]")
    n, b = Q.shape[0], Q.shape[1] // 16
    if n > 0x7FFFFFFF or 32 * b > 0x7FFFFFFF:
        raise ValueError(f"{name} has more than 2^31 - 1 rows or columns")
    _shaped(Q, torch.uint8, (n, 16 * b), name)
    _shaped(scales, torch.uint8, (n, b), its)
    return n, b


def quantize_mxfp4(X, Q=None, scales=None, stream=None):
    """(Q, scales): X ([n, F] float32 or bfloat16) in 4 bits (e2m1, two a byte, the first in the lower four bits) as uint8
    [n, 16 * ceil(F / 32)], with a scale 2^(s - 127) for each 32 consecutive features of a row, uint8
    [n, ceil(F / 32)] (255: NaN)."""
    flags = IN_BF16 if _rows(X, "X") else 0
    n, F = X.shape
    s = _queue(stream, X, Q, scales)
    Q, scales = _mx_out(X, n, F, Q, scales, stream)
    _check(_lib.dualgcn_quantize_mxfp4(X.data_ptr(), n, F, flags, Q.data_ptr(), scales.data_ptr(), s),
           "dualgcn_quantize_mxfp4")
    return Q, scales


def quantize_weight_mxfp4(W, transpose=True, Q=None, scales=None, stream=None):
    """(Q, scales): W ([F_in, F_out] float32) in 4 bits as update_mxfp4 reads it: F_out rows of F_in elements for X W, or
    with transpose=False F_in rows of F_out elements for the gradient's product G W^T (its blocks run along
    F_out: other numbers than the transposed form's)."""
    _dev(W, torch.float32, "W")
    if W.dim() != 2:
        raise ValueError("W must be [F_in, F_out]")
    F_in, F_out = W.shape
    if max(F_in, F_out) > 0x7FFFFFFF:
        raise ValueError("more than 2^31 - 1 rows or columns")
    s = _queue(stream, W, Q, scales)
    rows, F = (F_out, F_in) if transpose else (F_in, F_out)
    Q, scales = _mx_out(W, rows, F, Q, scales, stream)
    _check(_lib.dualgcn_quantize_weight_mxfp4(W.data_ptr(), F_in, F_out, 1 if transpose else 0, Q.data_ptr(),
                                              scales.data_ptr(), s), "dualgcn_quantize_weight_mxfp4")
    return Q, scales


def dequantize_mxfp4(Q, scales, F=None, X=None, out_bf16=False, stream=None):
    """The values of quantize_mxfp4's (Q, scales) as float32 [n, F], or bfloat16 with out_bf16 (both hold every one).
    F: the features of a row, where the last block is not full."""
    n, b = _mx(Q, scales, "Q", "scales")
    if F is None:
        F = 32 * b
    if _mx_blocks(F) != b or F < 1:
        raise ValueError(f"rows of {F} elements have {_mx_blocks(F)} blocks, not {b}")
    s = _queue(stream, Q, scales, X)
    xdt = torch.bfloat16 if out_bf16 else torch.float32
    X = _empty((n, F), xdt, Q, stream) if X is None else _shaped(X, xdt, (n, F), "X")
    _check(_lib.dualgcn_dequantize_mxfp4(Q.data_ptr(), scales.data_ptr(), n, F, OUT_BF16 if out_bf16 else 0, X.data_ptr(),
                                         s), "dualgcn_dequantize_mxfp4")
    return X


def update_mxfp4(X, sx, W, sw, T=None, out_bf16=False, stream=None):
    """T = X W from 4-bit operands on the matrix cores, both as quantize_mxfp4 and quantize_weight_mxfp4 make them: X uint8
    [n, 16 * blocks] with its scales sx [n, blocks], W uint8 [F_out, 16 * blocks] (transposed) with sw [F_out, blocks].
    T is float32 [n, F_out], or bfloat16 with out_bf16."""
    n, b = _mx(X, sx, "X", "sx")
    F_out, wb = _mx(W, sw, "W", "sw")
    if wb != b:
        raise ValueError(f"X has {b} blocks a row, W {wb}")
    s = _queue(stream, X, sx, W, sw, T)
    tdt = torch.bfloat16 if out_bf16 else torch.float32
    T = _empty((n, F_out), tdt, X, stream) if T is None else _shaped(T, tdt, (n, F_out), "T")
    _check(_lib.dualgcn_update_mxfp4(X.data_ptr(), sx.data_ptr(), W.data_ptr(), sw.data_ptr(), T.data_ptr(), n, 32 * b,
                                     F_out, OUT_BF16 if out_bf16 else 0, s), "dualgcn_update_mxfp4")
    return T


PROBE_COPY, PROBE_READ = 0, 1


def bandwidth_probe(kind, src, dst, stream=None):
    """dualgcn_bandwidth_probe: kind PROBE_COPY (dst = src) or PROBE_READ (src read once;
    dst receives per-workgroup sums, at least bandwidth_probe_out_floats() floats)."""
    nbytes = src.numel() * src.element_size()
    if kind == PROBE_COPY and dst.numel() * dst.element_size() < nbytes:
        raise ValueError("dst smaller than src")
    if kind == PROBE_READ and dst.numel() * dst.element_size() < 4 * _lib.dualgcn_bandwidth_probe_out_floats():
        raise ValueError("dst too small for the read probe's sums")
    _check(_lib.dualgcn_bandwidth_probe(kind, src.data_ptr(), dst.data_ptr(), nbytes, _stream(stream)),
           "dualgcn_bandwidth_probe")


def bandwidth_probe_out_floats():
    return int(_lib.dualgcn_bandwidth_probe_out_floats())


def arw_patterns(rowptr, col, val, seed, walks_per_node, walk_len, stream=None):
    """uint8 [n, k, d+1] anonymous walks (labels) of every node, on the device."""
    csr = make_csr(rowptr, col, val)
    out = torch.empty((csr.n, walks_per_node, walk_len + 1), dtype=torch.uint8,
                      device=rowptr.device)
    _check(_lib.dualgcn_arw_patterns(ctypes.byref(csr), seed, walks_per_node, walk_len,
                                     out.data_ptr(), _stream(stream)), "dualgcn_arw_patterns")
    return out


__all__ = ["Plan", "spmm", "spmm_update", "update", "gcn_layer", "gcn_layer_workspace_bytes", "arw_patterns",
           "DualGCNError", "lib", "status_str", "make_csr", "Csr", "Thresholds", "PlanInfo",
           "FORCE_AUTO", "FORCE_SPARSE", "FORCE_DENSE", "RELU", "OUT_BF16", "IN_BF16",
           "ALPHA_ADAPTIVE", "ALPHA_BALANCED", "GRAD_BF16", "LOSS_SLOTS", "softmax_xent", "weight_grad", "weight_grad_noalloc",
           "weight_grad_workspace_bytes", "backward_data", "aggregator_values", "AGG_GCN",
           "AGG_MEAN", "AGG_SUM", "bandwidth_probe", "bandwidth_probe_out_floats",
           "PROBE_COPY", "PROBE_READ", "norm_residual", "norm_residual_backward", "NormGrads",
           "norm_residual_backward_workspace_bytes", "Norm", "NormGradPointers", "STREAM_BF16", "NORM_LAYER",
           "NORM_POST", "GATE_FEATURE", "GATE_NODE", "GATE_FULL", "GATE_SIGMOID",
           "distill_xent", "distill_workspace_bytes", "TEACHER_BF16",
           "quantize_fp8", "quantize_weight_fp8", "update_fp8", "FP8_BLOCK",
           "group_norm", "group_norm_backward", "GroupNormGrads", "group_norm_workspace_bytes", "GroupNorm", "SILU",
           "ZERO_REST", "grad_norm", "clip_grads", "clipped_sgd", "grad_norm_workspace_bytes", "Grad",
           "quantize_mxfp4", "quantize_weight_mxfp4", "dequantize_mxfp4", "update_mxfp4", "MX_BLOCK"]
