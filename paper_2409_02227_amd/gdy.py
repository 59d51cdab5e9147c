"""ctypes binding of libgdy (include/gdy.h): argument marshalling only.

Every step of the hot path -- validation, features, CD prediction,
grouping, variant binding, launches -- runs inside libgdy.so.  This module
turns Python/torch objects into the C structures and back.  Loading fails
loudly when the library is missing; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgdy.so")

MAX_GEMMS = 256
N_CD = 5
N_FEATURES = 18
CD_CLASSES = (1, 2, 4, 8, 16)

# gdy_dtype
F16, BF16, FP8_E4M3, F32 = 1, 2, 3, 4
# gdy_mode
SEQUENTIAL, DEFAULT, GO, SELECTOR, FORCED, FORCED_GROUPED = 0, 1, 2, 3, 4, 5
CU_PARTITION, CU_PARTITION_GO, CU_PARTITION_RC = 6, 7, 8
GEMM, ADD = 0, 1  # gdy_op
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4  # gdy_act
ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}
OVER_ROWS, OVER_K = 0, 1  # gdy_over
MAX_GROUPS = 4096
MAX_TOP_K = 64
ROUTE_ALONE = 2048
MODES = {"sequential": SEQUENTIAL, "default": DEFAULT, "go": GO,
         "selector": SELECTOR, "forced": FORCED, "forced_grouped": FORCED_GROUPED,
         "cu_partition": CU_PARTITION, "cu_partition_go": CU_PARTITION_GO,
         "cu_partition_rc": CU_PARTITION_RC}
# gdy_create use_cu_masks bits
RC_STREAMS, PARTITION_STREAMS = 1, 2

STATUS = {0: "GDY_OK", 1: "GDY_ERR_INVALID_ARG", 2: "GDY_ERR_UNSUPPORTED", 3: "GDY_ERR_ALIAS",
          4: "GDY_ERR_TOO_MANY", 5: "GDY_ERR_TABLE", 6: "GDY_ERR_HIP", 7: "GDY_ERR_NOMEM"}

EXPORTS = ("gdy_create", "gdy_destroy", "gdy_set_rc", "gdy_plan", "gdy_execute", "gdy_execute_static",
           "gdy_execute_epilogue", "gdy_execute_epilogue_static", "gdy_execute_grouped", "gdy_grouped_tile",
           "gdy_execute_act_grad", "gdy_execute_route", "gdy_execute_scatter", "gdy_execute_combine",
           "gdy_execute_quantize", "gdy_execute_integer", "gdy_integer_tile",
           "gdy_set_timing", "gdy_last_kernel_times", "gdy_kernel_times", "gdy_features", "gdy_dispatch_map",
           "gdy_variant_count",
           "gdy_variant_info", "gdy_variant_find", "gdy_isolated_variant",
           "gdy_catalogue_hash", "gdy_device_cus", "gdy_status_string", "gdy_last_error")


class GemmDesc(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("a_type", ctypes.c_int32), ("b_type", ctypes.c_int32), ("c_type", ctypes.c_int32),
                ("trans_a", ctypes.c_int32), ("trans_b", ctypes.c_int32),
                ("a", ctypes.c_void_p), ("lda", ctypes.c_int64),
                ("b", ctypes.c_void_p), ("ldb", ctypes.c_int64),
                ("c", ctypes.c_void_p), ("ldc", ctypes.c_int64),
                ("scale_a", ctypes.c_float), ("scale_b", ctypes.c_float),
                ("tenant", ctypes.c_int32), ("variant", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("op", ctypes.c_int32),
                ("stride_a", ctypes.c_int64), ("stride_b", ctypes.c_int64),
                ("stride_c", ctypes.c_int64)]


class EpilogueDesc(ctypes.Structure):
    _fields_ = [("act", ctypes.c_int32), ("grad", ctypes.c_int32),
                ("bias", ctypes.c_void_p), ("bias_type", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("aux", ctypes.c_void_p), ("ldaux", ctypes.c_int64),
                ("bias_grad", ctypes.c_void_p),
                ("stride_bias", ctypes.c_int64), ("stride_r", ctypes.c_int64),
                ("stride_aux", ctypes.c_int64), ("stride_bias_grad", ctypes.c_int64)]


class GroupedDesc(ctypes.Structure):
    _fields_ = [("over", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("a_type", ctypes.c_int32), ("b_type", ctypes.c_int32), ("c_type", ctypes.c_int32),
                ("trans_b", ctypes.c_int32), ("offsets", ctypes.c_void_p),
                ("a", ctypes.c_void_p), ("lda", ctypes.c_int64),
                ("b", ctypes.c_void_p), ("ldb", ctypes.c_int64), ("stride_b", ctypes.c_int64),
                ("c", ctypes.c_void_p), ("ldc", ctypes.c_int64), ("stride_c", ctypes.c_int64),
                ("scale_a", ctypes.c_float), ("scale_b", ctypes.c_float), ("scales", ctypes.c_void_p)]


class ActGradDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("n", ctypes.c_int64), ("type", ctypes.c_int32), ("act", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("reserved", ctypes.c_int32), ("offsets", ctypes.c_void_p),
                ("dy", ctypes.c_void_p), ("lddy", ctypes.c_int64), ("z", ctypes.c_void_p), ("ldz", ctypes.c_int64),
                ("dz", ctypes.c_void_p), ("lddz", ctypes.c_int64),
                ("bias_grad", ctypes.c_void_p), ("stride_bias_grad", ctypes.c_int64)]


class RouteDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("top_k", ctypes.c_int32), ("experts", ctypes.c_int32),
                ("ids", ctypes.c_void_p), ("ld_ids", ctypes.c_int64),
                ("id_bytes", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("slots", ctypes.c_void_p), ("offsets", ctypes.c_void_p)]


class ScatterDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("rows", ctypes.c_int64), ("n", ctypes.c_int64),
                ("top_k", ctypes.c_int32), ("type", ctypes.c_int32), ("slots", ctypes.c_void_p),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("weights", ctypes.c_void_p),
                ("weights_type", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("out", ctypes.c_void_p), ("ldo", ctypes.c_int64), ("z", ctypes.c_void_p), ("ldz", ctypes.c_int64),
                ("weight_grad", ctypes.c_void_p)]


class CombineDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("rows", ctypes.c_int64), ("n", ctypes.c_int64),
                ("top_k", ctypes.c_int32), ("type", ctypes.c_int32), ("slots", ctypes.c_void_p),
                ("z", ctypes.c_void_p), ("ldz", ctypes.c_int64), ("weights", ctypes.c_void_p),
                ("weights_type", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64), ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64)]


class QuantizeDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("n", ctypes.c_int64), ("type", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("slots", ctypes.c_void_p),
                ("out_rows", ctypes.c_int64), ("q", ctypes.c_void_p), ("ldq", ctypes.c_int64),
                ("scales", ctypes.c_void_p)]


class IntegerDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("c_type", ctypes.c_int32), ("trans_b", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("reserved", ctypes.c_int32), ("offsets", ctypes.c_void_p),
                ("a", ctypes.c_void_p), ("lda", ctypes.c_int64),
                ("b", ctypes.c_void_p), ("ldb", ctypes.c_int64), ("stride_b", ctypes.c_int64),
                ("row_scales", ctypes.c_void_p), ("col_scales", ctypes.c_void_p),
                ("stride_col_scales", ctypes.c_int64), ("c", ctypes.c_void_p), ("ldc", ctypes.c_int64)]


class Plan(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("cd", ctypes.c_int32), ("n_groups", ctypes.c_int32),
                ("fallback", ctypes.c_int32),
                ("order", ctypes.c_int32 * MAX_GEMMS), ("group_of", ctypes.c_int32 * MAX_GEMMS),
                ("stream_of", ctypes.c_int32 * MAX_GEMMS), ("variant_of", ctypes.c_int32 * MAX_GEMMS),
                ("pred_cd", ctypes.c_int32 * MAX_GEMMS), ("group_size", ctypes.c_int32 * MAX_GEMMS),
                ("n_dispatches", ctypes.c_int32), ("dispatch_of", ctypes.c_int32 * MAX_GEMMS),
                ("split_of", ctypes.c_int32 * MAX_GEMMS)]

    def as_dict(self) -> dict:
        n = self.n
        return {"n": n, "cd": self.cd, "n_groups": self.n_groups, "fallback": self.fallback,
                "order": [x for x in self.order[:n] if x >= 0],
                "group_of": list(self.group_of[:n]), "stream_of": list(self.stream_of[:n]),
                "variant_of": list(self.variant_of[:n]), "pred_cd": list(self.pred_cd[:n]),
                "group_size": list(self.group_size[:self.n_groups]),
                "n_dispatches": self.n_dispatches, "dispatch_of": list(self.dispatch_of[:n]),
                "split_of": list(self.split_of[:n])}


class VariantDesc(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 64), ("dtype", ctypes.c_int32), ("trans_a", ctypes.c_int32),
                ("trans_b", ctypes.c_int32), ("bm", ctypes.c_int32), ("bn", ctypes.c_int32),
                ("bk", ctypes.c_int32), ("waves", ctypes.c_int32), ("mfma", ctypes.c_int32),
                ("lds_bytes", ctypes.c_int32), ("vgprs", ctypes.c_int32),
                ("occupancy", ctypes.c_int32), ("grid_cap_cus", ctypes.c_int32),
                ("direct", ctypes.c_int32), ("kind", ctypes.c_int32)]

    def as_dict(self) -> dict:
        d = {f: getattr(self, f) for f, _ in self._fields_}
        d["name"] = self.name.decode()
        return d


class GdyError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


_lib = None


def load_library(path: str = None) -> ctypes.CDLL:
    """Load libgdy.so (raises if it is missing: no fallback exists).
    GDY_LIBRARY names another build of it (the sanitizer build)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or os.environ.get("GDY_LIBRARY") or LIB_PATH
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with paper_2409_02227_amd.build.build()")
    lib = ctypes.CDLL(path)
    P, i32, i64, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64
    sig = {
        "gdy_create": (i32, [ctypes.POINTER(P), ctypes.c_int, ctypes.c_char_p, i32, i32]),
        "gdy_destroy": (None, [P]),
        "gdy_set_rc": (i32, [P, i32]),
        "gdy_plan": (i32, [P, ctypes.POINTER(GemmDesc), i32, i32, i32, ctypes.POINTER(Plan)]),
        "gdy_execute": (i32, [P, ctypes.POINTER(GemmDesc), i32, i32, i32, P, ctypes.POINTER(Plan)]),
        "gdy_execute_static": (i32, [P, ctypes.POINTER(GemmDesc), i32, i32, i32, P, ctypes.POINTER(Plan)]),
        "gdy_execute_epilogue": (i32, [P, ctypes.POINTER(GemmDesc), ctypes.POINTER(EpilogueDesc), i32, i32, i32, P,
                                       ctypes.POINTER(Plan)]),
        "gdy_execute_epilogue_static": (i32, [P, ctypes.POINTER(GemmDesc), ctypes.POINTER(EpilogueDesc), i32, i32,
                                              i32, P, ctypes.POINTER(Plan)]),
        "gdy_execute_grouped": (i32, [P, ctypes.POINTER(GroupedDesc), ctypes.POINTER(EpilogueDesc), P]),
        "gdy_grouped_tile": (i32, [P, ctypes.POINTER(GroupedDesc), ctypes.POINTER(i32), ctypes.POINTER(i32)]),
        "gdy_execute_act_grad": (i32, [P, ctypes.POINTER(ActGradDesc), P]),
        "gdy_execute_route": (i32, [P, ctypes.POINTER(RouteDesc), P]),
        "gdy_execute_scatter": (i32, [P, ctypes.POINTER(ScatterDesc), P]),
        "gdy_execute_combine": (i32, [P, ctypes.POINTER(CombineDesc), P]),
        "gdy_execute_quantize": (i32, [P, ctypes.POINTER(QuantizeDesc), P]),
        "gdy_execute_integer": (i32, [P, ctypes.POINTER(IntegerDesc), ctypes.POINTER(EpilogueDesc), P]),
        "gdy_integer_tile": (i32, [P, ctypes.POINTER(IntegerDesc), ctypes.POINTER(i32), ctypes.POINTER(i32)]),
        "gdy_set_timing": (i32, [P, i32]),
        "gdy_last_kernel_times": (i32, [P, ctypes.POINTER(ctypes.c_float),
                                        ctypes.POINTER(ctypes.c_float), i32]),
        "gdy_kernel_times": (i32, [P, i32, ctypes.POINTER(ctypes.c_float),
                                   ctypes.POINTER(ctypes.c_float), i32]),
        "gdy_features": (i32, [P, ctypes.POINTER(GemmDesc), ctypes.POINTER(ctypes.c_double)]),
        "gdy_dispatch_map": (i32, [P, ctypes.POINTER(GemmDesc), i32, i32, i32, i32, i32, ctypes.POINTER(i32),
                                   ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                   ctypes.POINTER(i64)]),
        "gdy_variant_count": (i32, [P]),
        "gdy_variant_info": (i32, [P, i32, ctypes.POINTER(VariantDesc)]),
        "gdy_variant_find": (i32, [P, ctypes.c_char_p]),
        "gdy_isolated_variant": (i32, [P, ctypes.POINTER(GemmDesc)]),
        "gdy_catalogue_hash": (u64, [P]),
        "gdy_device_cus": (i32, [P]),
        "gdy_status_string": (ctypes.c_char_p, [i32]),
        "gdy_last_error": (ctypes.c_char_p, [P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


_TORCH_DTYPE = None


def _dtype_code(t) -> int:
    global _TORCH_DTYPE
    if _TORCH_DTYPE is None:
        import torch
        _TORCH_DTYPE = {torch.float16: F16, torch.bfloat16: BF16, torch.float8_e4m3fn: FP8_E4M3,
                        torch.uint8: FP8_E4M3, torch.float32: F32}
    return _TORCH_DTYPE[t.dtype]


def _rows_of(t, name="operands"):
    """A matrix's leading dimension; its rows must be contiguous and lie apart."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D (or 3-D batches) with a contiguous last dimension")
    if t.shape[0] > 1 and t.stride(0) < 1:  # an expanded matrix: no leading dimension reads one row again
        raise ValueError(f"the rows of {name} must not be one row expanded")
    if t.shape[0] <= 1:  # a single row's stride says nothing
        return max(t.stride(0), t.shape[1], 1)
    return t.stride(0)


@dataclass
class Add:
    """Element-wise C = A + B over an M x N region: the non-GEMM that co-runs
    with GEMMs (Sec. 7.1).  2-D tensors of one type (bf16, fp16, fp32), or
    3-D strided batches; the last dimension contiguous."""
    a: object
    b: object
    c: object
    tenant: int = 0
    variant: int = -1

    def desc(self) -> GemmDesc:
        a, b, c = self.a, self.b, self.c
        batch = c.shape[0] if c.dim() == 3 else 0
        if batch and any(t.dim() == 3 and t.shape[0] != batch for t in (a, b)):
            raise ValueError("batched operands disagree on the batch size")
        if not batch and (a.dim() == 3 or b.dim() == 3):
            raise ValueError("a batched A or B needs a batched C")

        def mat(t):
            return (t[0], t.stride(0)) if t.dim() == 3 else (t, 0)
        (a2, sa), (b2, sb), (c2, sc) = mat(a), mat(b), mat(c)
        lda, ldb, ldc = _rows_of(a2), _rows_of(b2), _rows_of(c2)
        m, n = c2.shape
        if tuple(a2.shape) != (m, n) or tuple(b2.shape) != (m, n):
            raise ValueError("add operands must have C's shape")
        d = GemmDesc()
        d.m, d.n, d.k = m, n, 0
        d.a_type, d.b_type, d.c_type = _dtype_code(a), _dtype_code(b), _dtype_code(c)
        d.a, d.lda = a.data_ptr(), lda
        d.b, d.ldb = b.data_ptr(), ldb
        d.c, d.ldc = c.data_ptr(), ldc
        d.scale_a = d.scale_b = 1.0
        d.tenant, d.variant = int(self.tenant), int(self.variant)
        d.batch, d.op = batch, ADD
        d.stride_a, d.stride_b, d.stride_c = sa, sb, sc
        return d


def _check_device(device, what, *tensors):
    """An address of another device's memory, or of the host's, faults in a kernel (device
    < 0, a host-only context: nothing is read)."""
    for t in tensors:
        if t is not None and device >= 0 and t.get_device() != device:
            raise ValueError(f"{what}: a tensor on {t.device}, the context is on cuda:{device}")


def _act(act) -> int:
    if isinstance(act, str):
        if act not in ACTS:
            raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTS)}")
        return ACTS[act]
    return int(act)


def _check_offsets(offsets):
    import torch
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or not offsets.is_contiguous() or offsets.shape[0] < 1:
        raise ValueError("offsets must be a contiguous int32 vector of groups + 1 values")
    return offsets.shape[0] - 1


def _bias_grad_stride(t, n, items):
    """bias_grad: fp32, n values (summed over the items) or items x n."""
    import torch
    if t.dtype != torch.float32:
        raise ValueError("bias_grad must be fp32")
    if t.dim() == 1 and tuple(t.shape) == (n,) and (n < 2 or t.stride(0) == 1):
        return 0
    if t.dim() == 2 and tuple(t.shape) == (items, n) and (n < 2 or t.stride(1) == 1):
        if items > 1 and t.stride(0) == 0:
            raise ValueError("the rows of bias_grad must not be one row expanded")
        return t.stride(0) if items > 1 else 0
    raise ValueError(f"bias_grad must hold {n} or {items} x {n} values, rows contiguous")


@dataclass
class Epilogue:
    """What a GEMM does with its sums before their rounding (gdy_epilogue):
    z = sums + bias, aux = z, C = act(z) + residual; with grad, from the saved
    pre-activation aux, C = (sums + bias) * act'(aux) + residual.

    bias: N values of C's type or fp32 (batch x N, or groups x N: one for each
    item).  residual, aux: of C's shape and type.  bias_grad: fp32, overwritten with
    the column sums of the unrounded C (N values, or batch x N / groups x N).
    act: none, relu, gelu, gelu_tanh or silu."""
    bias: object = None
    act: object = "none"
    residual: object = None
    aux: object = None
    grad: bool = False
    bias_grad: object = None

    def tensors(self):
        return self.bias, self.residual, self.aux, self.bias_grad

    def desc(self, c, items: int = 0) -> EpilogueDesc:
        """For the output tensor c; items: batch items of a 3-D c, or the groups
        that bias and bias_grad may be given for."""
        e = EpilogueDesc()
        e.act, e.grad = _act(self.act), int(bool(self.grad))
        n = c.shape[-1]
        if self.bias is not None:
            b = self.bias
            if tuple(b.shape) == (n,):
                e.stride_bias = 0
            elif items and tuple(b.shape) == (items, n):
                e.stride_bias = b.stride(0) if items > 1 else 0
            else:
                raise ValueError(f"bias must hold {n} values" + (f" or {items} x {n}" if items else ""))
            if n > 1 and b.stride(-1) != 1:
                raise ValueError("bias must be contiguous")
            e.bias, e.bias_type = b.data_ptr(), _dtype_code(b)
        for name, ld, stride in (("residual", "ldr", "stride_r"), ("aux", "ldaux", "stride_aux")):
            t = getattr(self, name)
            if t is None:
                continue
            if t.dtype != c.dtype or tuple(t.shape) != tuple(c.shape):
                raise ValueError(f"{name} must have C's shape and type")
            setattr(e, name, t.data_ptr())
            setattr(e, ld, _rows_of(t[0] if t.dim() == 3 else t, name) if t.dim() == 2 or t.shape[0] else 1)
            setattr(e, stride, t.stride(0) if t.dim() == 3 else 0)
        if self.bias_grad is not None:
            e.stride_bias_grad = _bias_grad_stride(self.bias_grad, n, max(items, 1))
            e.bias_grad = self.bias_grad.data_ptr()
        return e


@dataclass
class Grouped:
    """One product grouped by expert (gdy_grouped).  The rows of a are sorted by
    group, group e holding rows offsets[e] to offsets[e + 1] (int32, on the device).

    over "rows": c (rows x N) = a (rows x K) times b[e] (groups x K x N, or groups x
    N x K with trans_b).  over "k": c[e] (groups x K x N) = a[e]^T b[e], the rows of e
    of a (rows x K) and b (rows x N).  scales: one fp32 scale a group (fp8)."""
    a: object
    b: object
    c: object
    offsets: object
    over: str = "rows"
    trans_b: int = 0
    scale_a: float = 1.0
    scale_b: float = 1.0
    scales: object = None
    epilogue: object = None

    def tensors(self):
        return (self.a, self.b, self.c, self.offsets, self.scales) + (self.epilogue.tensors() if self.epilogue else ())

    def descs(self):
        """(GroupedDesc, EpilogueDesc or None)."""
        import torch
        a, b, c = self.a, self.b, self.c
        d = GroupedDesc()
        groups = d.groups = _check_offsets(self.offsets)
        if self.over not in ("rows", "k"):
            raise ValueError("over must be 'rows' or 'k'")
        over_k = self.over == "k"
        d.over = OVER_K if over_k else OVER_ROWS
        per_group = c if over_k else b
        if per_group.dim() != 3 or per_group.shape[0] != groups:
            raise ValueError(f"{'c' if over_k else 'b'} must be a 3-D tensor of {groups} groups")
        if a.dim() != 2 or (b if over_k else c).dim() != 2:
            raise ValueError("the row matrices must be 2-D")
        d.rows, d.k = a.shape
        d.trans_b = int(self.trans_b)
        if over_k:
            d.n = b.shape[1]
            ok = b.shape[0] == d.rows and tuple(c.shape[1:]) == (d.k, d.n)
        else:
            d.n = c.shape[1]
            ok = c.shape[0] == d.rows and tuple(b.shape[1:]) == ((d.n, d.k) if d.trans_b else (d.k, d.n))
        if not ok:
            raise ValueError(f"shapes disagree: a {tuple(a.shape)}, b {tuple(b.shape)}, c {tuple(c.shape)}")
        d.a_type, d.b_type, d.c_type = _dtype_code(a), _dtype_code(b), _dtype_code(c)
        d.offsets = self.offsets.data_ptr()

        def item(t, name):
            if t.dim() == 3:
                return (_rows_of(t[0], name) if groups else 1), t.stride(0)
            return _rows_of(t, name), 0
        d.a, (d.lda, _) = a.data_ptr(), item(a, "a")
        d.b, (d.ldb, d.stride_b) = b.data_ptr(), item(b, "b")
        d.c, (d.ldc, d.stride_c) = c.data_ptr(), item(c, "c")
        d.scale_a, d.scale_b = float(self.scale_a), float(self.scale_b)
        if self.scales is not None:
            if self.scales.dtype != torch.float32 or tuple(self.scales.shape) != (groups,) or \
                    not self.scales.is_contiguous():
                raise ValueError("scales must hold one fp32 value a group")
            d.scales = self.scales.data_ptr()
        return d, (None if self.epilogue is None else self.epilogue.desc(c, groups))


@dataclass
class ActGrad:
    """dz = dy * act'(z) and bias_grad = the column sums of dy * act'(z) (gdy_act_grad),
    over all rows, or with offsets (int32, groups + 1) over the rows of each group.
    z may be None where act is none; dz or bias_grad may be None."""
    dy: object
    z: object = None
    dz: object = None
    bias_grad: object = None
    act: object = "none"
    offsets: object = None

    def tensors(self):
        return self.dy, self.z, self.dz, self.bias_grad, self.offsets

    def desc(self) -> ActGradDesc:
        d = ActGradDesc()
        if self.dy.dim() != 2:
            raise ValueError("dy must be 2-D")
        d.rows, d.n = self.dy.shape
        d.type, d.act = _dtype_code(self.dy), _act(self.act)
        if d.act != ACT_NONE and self.z is None:
            raise ValueError("an activation needs z")
        for name in ("dy", "z", "dz"):
            t = getattr(self, name)
            if t is None:
                continue
            if t.dtype != self.dy.dtype or tuple(t.shape) != tuple(self.dy.shape):
                raise ValueError(f"{name} must have dy's shape and type")
            setattr(d, name, t.data_ptr())
            setattr(d, "ld" + name, _rows_of(t, name))
        if self.offsets is not None:
            d.groups = _check_offsets(self.offsets)
            d.offsets = self.offsets.data_ptr()
        if self.bias_grad is not None:
            d.stride_bias_grad = _bias_grad_stride(self.bias_grad, d.n, max(d.groups, 1))
            d.bias_grad = self.bias_grad.data_ptr()
        return d


def _matrix(t, name, dtype=None, cols=None):
    """(rows, columns, leading dimension) of a 2-D tensor."""
    if t.dim() != 2 or (cols is not None and t.shape[1] != cols) or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be 2-D" + (f" with {cols} columns" if cols is not None else "") +
                         (f" of {dtype}" if dtype is not None else ""))
    return t.shape[0], t.shape[1], _rows_of(t, name)


def _row_dtype(t, name) -> int:
    """The code of a floating type; uint8 is not taken for fp8 here."""
    import torch
    codes = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32, torch.float8_e4m3fn: FP8_E4M3}
    if t.dtype not in codes:
        raise ValueError(f"{name} of {t.dtype}")
    return codes[t.dtype]


def _check_slots(slots, tokens):
    import torch
    if slots.dtype != torch.int32 or slots.dim() != 2 or slots.shape[0] != tokens or not slots.is_contiguous():
        raise ValueError(f"slots must be a contiguous int32 matrix of {tokens} rows")
    return slots.shape[1]


def _pair_weights(d, weights, slots, like):
    """The fields of the weights of pairs: fp32 or of the rows' type."""
    import torch
    if weights is None:
        return
    if tuple(weights.shape) != tuple(slots.shape) or not weights.is_contiguous() or \
            weights.dtype not in (torch.float32, like.dtype):
        raise ValueError("weights must be contiguous, of the slots' shape, fp32 or of the rows' type")
    d.weights, d.weights_type = weights.data_ptr(), _row_dtype(weights, "weights")


@dataclass
class Route:
    """The rows of each expert (gdy_route): from ids (tokens x top_k, int32 or int64, on the
    device; outside 0 .. experts - 1: none) the slots of the pairs (tokens x top_k, int32)
    and the bounds of the experts' rows, offsets (experts + 1, int32)."""
    ids: object
    slots: object
    offsets: object

    def tensors(self):
        return self.ids, self.slots, self.offsets

    def desc(self) -> RouteDesc:
        import torch
        d = RouteDesc()
        if self.ids.dtype not in (torch.int32, torch.int64):
            raise ValueError("ids must be int32 or int64")
        d.tokens, d.top_k, d.ld_ids = _matrix(self.ids, "ids")
        if _check_slots(self.slots, d.tokens) != d.top_k:
            raise ValueError("slots must have the ids' shape")
        d.experts = _check_offsets(self.offsets)
        d.id_bytes = self.ids.element_size()
        d.ids, d.slots, d.offsets = self.ids.data_ptr(), self.slots.data_ptr(), self.offsets.data_ptr()
        return d


@dataclass
class Scatter:
    """Rows to the experts (gdy_scatter): out[slots[t, j]] = weights[t, j] * x[t] (weights None: x[t] itself).
    weight_grad (fp32, of the slots' shape): the sums of x[t] * z[slots[t, j]], z of out's shape; with x
    the gradient of a Combine's y, out and weight_grad are those of its z and weights."""
    x: object
    slots: object
    out: object
    weights: object = None
    z: object = None
    weight_grad: object = None

    def tensors(self):
        return self.x, self.slots, self.out, self.weights, self.z, self.weight_grad

    def desc(self) -> ScatterDesc:
        import torch
        d = ScatterDesc()
        d.type = _row_dtype(self.x, "x")
        d.tokens, d.n, d.ldx = _matrix(self.x, "x")
        d.rows, _, d.ldo = _matrix(self.out, "out", self.x.dtype, d.n)
        d.top_k = _check_slots(self.slots, d.tokens)
        d.slots, d.x, d.out = self.slots.data_ptr(), self.x.data_ptr(), self.out.data_ptr()
        _pair_weights(d, self.weights, self.slots, self.x)
        if (self.weight_grad is None) != (self.z is None) or (self.z is not None and self.weights is None):
            raise ValueError("z and weight_grad belong together, and need weights")
        if self.z is not None:
            if _matrix(self.z, "z", self.x.dtype, d.n)[0] != d.rows:
                raise ValueError("z must have out's shape")
            d.z, d.ldz = self.z.data_ptr(), _rows_of(self.z, "z")
            g = self.weight_grad
            if g.dtype != torch.float32 or tuple(g.shape) != tuple(self.slots.shape) or not g.is_contiguous():
                raise ValueError("weight_grad must be contiguous fp32 of the slots' shape")
            d.weight_grad = g.data_ptr()
        return d


@dataclass
class Combine:
    """Rows back from the experts (gdy_combine): y[t] = sum over j of weights[t, j] * z[slots[t, j]], plus residual[t].
    weights None: their sum, the gradient of a Scatter's x.  residual may be y."""
    z: object
    slots: object
    y: object
    weights: object = None
    residual: object = None

    def tensors(self):
        return self.z, self.slots, self.y, self.weights, self.residual

    def desc(self) -> CombineDesc:
        d = CombineDesc()
        d.type = _row_dtype(self.y, "y")
        d.tokens, d.n, d.ldy = _matrix(self.y, "y")
        d.rows, _, d.ldz = _matrix(self.z, "z", self.y.dtype, d.n)
        d.top_k = _check_slots(self.slots, d.tokens)
        d.slots, d.z, d.y = self.slots.data_ptr(), self.z.data_ptr(), self.y.data_ptr()
        _pair_weights(d, self.weights, self.slots, self.y)
        if self.residual is not None:
            if _matrix(self.residual, "residual", self.y.dtype, d.n)[0] != d.tokens:
                raise ValueError("residual must have y's shape")
            d.residual, d.ldr = self.residual.data_ptr(), _rows_of(self.residual, "residual")
        return d


@dataclass
class Quantize:
    """Rows in 8-bit integers (gdy_quantize): scales[i] = max |x[i]| / 127 (fp32), q[i] = x[i] / scales[i] to the
    nearest integer (int8).  slots (rows x top_k): row i goes to the rows slots[i] of q and scales."""
    x: object
    q: object
    scales: object
    slots: object = None

    def tensors(self):
        return self.x, self.q, self.scales, self.slots

    def desc(self) -> QuantizeDesc:
        import torch
        d = QuantizeDesc()
        d.type = _row_dtype(self.x, "x")
        d.rows, d.n, d.ldx = _matrix(self.x, "x")
        out_rows, _, d.ldq = _matrix(self.q, "q", torch.int8, d.n)
        if self.scales.dtype != torch.float32 or tuple(self.scales.shape) != (out_rows,) or \
                not self.scales.is_contiguous():
            raise ValueError("scales must hold one fp32 value a row of q")
        if self.slots is not None:
            top_k = _check_slots(self.slots, d.rows)
            if d.rows:  # without rows there are no slots either, and their address is null
                d.top_k, d.out_rows, d.slots = top_k, out_rows, self.slots.data_ptr()
        elif out_rows != d.rows:
            raise ValueError("q must have x's shape")
        d.x, d.q, d.scales = self.x.data_ptr(), self.q.data_ptr(), self.scales.data_ptr()
        return d


@dataclass
class Int8:
    """A product of 8-bit integers (gdy_integer): c = act(row_scales[i] * col_scales[j] * (a op(b))[i, j] + bias) +
    residual, a (rows x K) and b (K x N, or N x K with trans_b) int8, the sums exact, c bf16, fp16 or fp32.
    row_scales (rows) and col_scales (N): fp32, None: 1.  With offsets (int32, groups + 1) a product
    grouped by expert over rows, as Grouped: b is 3-D, col_scales and bias N or groups x N."""
    a: object
    b: object
    c: object
    row_scales: object = None
    col_scales: object = None
    offsets: object = None
    trans_b: int = 0
    epilogue: object = None

    def tensors(self):
        return (self.a, self.b, self.c, self.row_scales, self.col_scales, self.offsets) + \
            (self.epilogue.tensors() if self.epilogue else ())

    def descs(self):
        """(IntegerDesc, EpilogueDesc or None)."""
        import torch
        a, b, c = self.a, self.b, self.c
        d = IntegerDesc()
        d.rows, d.k, d.lda = _matrix(a, "a", torch.int8)
        d.n = c.shape[-1]
        if _matrix(c, "c")[0] != d.rows:
            raise ValueError("c must have a's rows")
        d.ldc, d.c_type = _rows_of(c, "c"), _row_dtype(c, "c")
        d.trans_b = int(self.trans_b)
        groups = 0
        if self.offsets is not None:
            groups = d.groups = _check_offsets(self.offsets)
            d.offsets = self.offsets.data_ptr()
        want = ((groups,) if self.offsets is not None else ()) + ((d.n, d.k) if d.trans_b else (d.k, d.n))
        if b.dtype != torch.int8 or tuple(b.shape) != want:
            raise ValueError(f"b must be int8 of shape {want}")
        if b.dim() == 3:
            d.ldb, d.stride_b = (_rows_of(b[0], "b") if groups else 1), b.stride(0)
        else:
            d.ldb = _rows_of(b, "b")
        d.a, d.b, d.c = a.data_ptr(), b.data_ptr(), c.data_ptr()
        for name, t, shapes in (("row_scales", self.row_scales, [(d.rows,)]),
                                ("col_scales", self.col_scales, [(d.n,)] + ([(groups, d.n)] if groups else []))):
            if t is None:
                continue
            if t.dtype != torch.float32 or tuple(t.shape) not in shapes or (t.shape[-1] > 1 and t.stride(-1) != 1):
                raise ValueError(f"{name} must be fp32 of shape {' or '.join(map(str, shapes))}, contiguous")
            setattr(d, name, t.data_ptr())
            if t.dim() == 2 and groups > 1:
                d.stride_col_scales = t.stride(0)
        return d, (None if self.epilogue is None else self.epilogue.desc(c, groups))


@dataclass
class Gemm:
    """One GEMM of a submission, from torch device tensors.

    a: M x K (or K x M when trans_a) row-major; b: K x N (or N x K when
    trans_b); c: M x N output.  Strided 2-D views are allowed as long as the
    last dimension is contiguous (ld = stride(0)).  A strided batch
    (B-GEMM) passes 3-D tensors whose first dimension is the batch: C must
    be 3-D; A or B may stay 2-D to be shared by every item (stride 0).
    epilogue: an Epilogue, or None."""
    a: object
    b: object
    c: object
    trans_a: int = 0
    trans_b: int = 0
    scale_a: float = 1.0
    scale_b: float = 1.0
    tenant: int = 0
    variant: int = -1
    epilogue: object = None

    def desc(self) -> GemmDesc:
        a, b, c = self.a, self.b, self.c
        batch = c.shape[0] if c.dim() == 3 else 0
        if batch and any(t.dim() == 3 and t.shape[0] != batch for t in (a, b)):
            raise ValueError("batched operands disagree on the batch size")
        if not batch and (a.dim() == 3 or b.dim() == 3):
            raise ValueError("a batched A or B needs a batched C")

        def mat(t):  # the 2-D item view and the item stride in elements
            if t.dim() == 3:
                return t[0], t.stride(0)
            return t, 0
        (a2, sa), (b2, sb), (c2, sc) = mat(a), mat(b), mat(c)
        lda, ldb, ldc = _rows_of(a2), _rows_of(b2), _rows_of(c2)
        m, n = c2.shape
        k = a2.shape[0] if self.trans_a else a2.shape[1]
        am = a2.shape[1] if self.trans_a else a2.shape[0]
        bk, bn = (b2.shape[1], b2.shape[0]) if self.trans_b else (b2.shape[0], b2.shape[1])
        if am != m or bn != n or bk != k:
            raise ValueError(f"shapes disagree: op(A) {am}x{k}, op(B) {bk}x{bn}, C {m}x{n}")
        d = GemmDesc()
        d.m, d.n, d.k = m, n, k
        d.a_type, d.b_type, d.c_type = _dtype_code(a), _dtype_code(b), _dtype_code(c)
        d.trans_a, d.trans_b = int(self.trans_a), int(self.trans_b)
        d.a, d.lda = a.data_ptr(), lda
        d.b, d.ldb = b.data_ptr(), ldb
        d.c, d.ldc = c.data_ptr(), ldc
        d.scale_a, d.scale_b = float(self.scale_a), float(self.scale_b)
        d.tenant, d.variant = int(self.tenant), int(self.variant)
        d.batch = batch
        d.stride_a, d.stride_b, d.stride_c = sa, sb, sc
        return d


def descs(gemms) -> ctypes.Array:
    """Marshal Gemm objects (or GemmDesc) into a C array once."""
    arr = (GemmDesc * max(len(gemms), 1))()
    for i, g in enumerate(gemms):
        arr[i] = g if isinstance(g, GemmDesc) else g.desc()
    return arr


def epilogue_descs(gemms):
    """The epilogues of a submission as a C array beside descs(gemms), or None
    where no member has one."""
    if not any(getattr(g, "epilogue", None) is not None for g in gemms):
        return None
    arr = (EpilogueDesc * max(len(gemms), 1))()
    for i, g in enumerate(gemms):
        e = getattr(g, "epilogue", None)
        if e is not None:
            arr[i] = e.desc(g.c, g.c.shape[0] if g.c.dim() == 3 else 0)
    return arr


class Context:
    """A libgdy context on one device (see gdy_create)."""

    def __init__(self, device: int = 0, table: str | None = None, max_streams: int = 16,
                 use_cu_masks: int = 0):
        self.lib = load_library()
        h = ctypes.c_void_p()
        st = self.lib.gdy_create(ctypes.byref(h), device,
                                 table.encode() if table else None, max_streams, int(use_cu_masks))
        if st != 0:
            raise GdyError(st, f"gdy_create failed (see stderr); table={table}")
        self.h = h
        self.device = device

    def close(self):
        if getattr(self, "h", None):
            self.lib.gdy_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_error(self) -> str:
        """gdy_last_error: the message of the last failure (after creation:
        why a GO table was not used), "" if none."""
        return self.lib.gdy_last_error(self.h).decode()

    def _check(self, st):
        if st != 0:
            raise GdyError(st, self.lib.gdy_last_error(self.h).decode())

    def plan(self, gemms, mode="selector", forced_cd: int = 0) -> dict:
        arr = descs(gemms)
        p = Plan()
        self._check(self.lib.gdy_plan(self.h, arr, len(gemms), _mode(mode), forced_cd, ctypes.byref(p)))
        return p.as_dict()

    def _stream_device(self):
        return self.device if self.device >= 0 else None

    def _epilogue_descs(self, gemms):
        """epilogue_descs() of members whose tensors all lie on the context's device."""
        eps = epilogue_descs(gemms)
        if eps is not None:
            for g in gemms:
                e = getattr(g, "epilogue", None)
                if e is not None:
                    _check_device(self.device, "a GEMM with an epilogue", g.a, g.b, g.c, *e.tensors())
        return eps

    def execute(self, gemms, mode="selector", forced_cd: int = 0, stream=None, want_plan=False):
        """Launch a submission on `stream` (torch stream, raw handle or None for
        torch's current stream of the context's device).  Returns the plan dict when want_plan.  Gemm
        objects may carry epilogues."""
        arr, eps = descs(gemms), self._epilogue_descs(gemms)
        handle = _stream_handle(stream, self._stream_device())
        p = Plan()
        if eps is None:
            self._check(self.lib.gdy_execute(self.h, arr, len(gemms), _mode(mode), forced_cd,
                                             handle, ctypes.byref(p)))
        else:
            self._check(self.lib.gdy_execute_epilogue(self.h, arr, eps, len(gemms), _mode(mode), forced_cd,
                                                      handle, ctypes.byref(p)))
        return p.as_dict() if want_plan else None

    def execute_static(self, gemms, mode="selector", forced_cd: int = 0, stream=None, want_plan=False):
        """gdy_execute_static: as execute(), with the split-K planes in the
        library's static device array (no allocation)."""
        arr, eps = descs(gemms), self._epilogue_descs(gemms)
        handle = _stream_handle(stream, self._stream_device())
        p = Plan()
        if eps is None:
            self._check(self.lib.gdy_execute_static(self.h, arr, len(gemms), _mode(mode), forced_cd,
                                                    handle, ctypes.byref(p)))
        else:
            self._check(self.lib.gdy_execute_epilogue_static(self.h, arr, eps, len(gemms), _mode(mode), forced_cd,
                                                             handle, ctypes.byref(p)))
        return p.as_dict() if want_plan else None

    def execute_descs(self, arr, n, mode, forced_cd, handle, epilogues=None):
        """Launch prepared GemmDesc arrays (no per-call marshalling); epilogues: as
        epilogue_descs() makes them."""
        if epilogues is None:
            self._check(self.lib.gdy_execute(self.h, arr, n, mode, forced_cd, handle, None))
        else:
            self._check(self.lib.gdy_execute_epilogue(self.h, arr, epilogues, n, mode, forced_cd, handle, None))

    def execute_grouped(self, product: Grouped, stream=None):
        """Launch a product grouped by expert (gdy_execute_grouped)."""
        _check_device(self.device, "a grouped product", *product.tensors())
        self.execute_grouped_descs(*product.descs(), _stream_handle(stream, self._stream_device()))

    def execute_grouped_descs(self, desc, epilogue, handle):
        """Launch a prepared GroupedDesc (epilogue: an EpilogueDesc or None)."""
        self._check(self.lib.gdy_execute_grouped(self.h, ctypes.byref(desc),
                                                 None if epilogue is None else ctypes.byref(epilogue), handle))

    def grouped_tile(self, product):
        """(rows, columns) of the tile that a Grouped or GroupedDesc runs on (gdy_grouped_tile)."""
        d = product if isinstance(product, GroupedDesc) else product.descs()[0]
        rows, cols = ctypes.c_int32(), ctypes.c_int32()
        self._check(self.lib.gdy_grouped_tile(self.h, ctypes.byref(d), ctypes.byref(rows), ctypes.byref(cols)))
        return rows.value, cols.value

    def execute_act_grad(self, op: ActGrad, stream=None):
        """Launch an activation and bias gradient (gdy_execute_act_grad)."""
        _check_device(self.device, "an activation gradient", *op.tensors())
        self.execute_act_grad_desc(op.desc(), _stream_handle(stream, self._stream_device()))

    def execute_act_grad_desc(self, desc, handle):
        """Launch a prepared ActGradDesc."""
        self._check(self.lib.gdy_execute_act_grad(self.h, ctypes.byref(desc), handle))

    def execute_route(self, op: Route, stream=None):
        """Launch a routing (gdy_execute_route)."""
        _check_device(self.device, "a routing", *op.tensors())
        self.execute_route_desc(op.desc(), _stream_handle(stream, self._stream_device()))

    def execute_route_desc(self, desc, handle):
        """Launch a prepared RouteDesc."""
        self._check(self.lib.gdy_execute_route(self.h, ctypes.byref(desc), handle))

    def execute_scatter(self, op: Scatter, stream=None):
        """Launch rows to the experts (gdy_execute_scatter)."""
        _check_device(self.device, "a scatter", *op.tensors())
        self.execute_scatter_desc(op.desc(), _stream_handle(stream, self._stream_device()))

    def execute_scatter_desc(self, desc, handle):
        """Launch a prepared ScatterDesc."""
        self._check(self.lib.gdy_execute_scatter(self.h, ctypes.byref(desc), handle))

    def execute_combine(self, op: Combine, stream=None):
        """Launch rows back from the experts (gdy_execute_combine)."""
        _check_device(self.device, "a combine", *op.tensors())
        self.execute_combine_desc(op.desc(), _stream_handle(stream, self._stream_device()))

    def execute_combine_desc(self, desc, handle):
        """Launch a prepared CombineDesc."""
        self._check(self.lib.gdy_execute_combine(self.h, ctypes.byref(desc), handle))

    def execute_quantize(self, op: Quantize, stream=None):
        """Launch rows to 8-bit integers (gdy_execute_quantize)."""
        _check_device(self.device, "a quantisation", *op.tensors())
        self.execute_quantize_desc(op.desc(), _stream_handle(stream, self._stream_device()))

    def execute_quantize_desc(self, desc, handle):
        """Launch a prepared QuantizeDesc."""
        self._check(self.lib.gdy_execute_quantize(self.h, ctypes.byref(desc), handle))

    def execute_int8(self, product: Int8, stream=None):
        """Launch a product of 8-bit integers (gdy_execute_integer)."""
        _check_device(self.device, "a product of 8-bit integers", *product.tensors())
        self.execute_int8_descs(*product.descs(), _stream_handle(stream, self._stream_device()))

    def execute_int8_descs(self, desc, epilogue, handle):
        """Launch a prepared IntegerDesc (epilogue: an EpilogueDesc or None)."""
        self._check(self.lib.gdy_execute_integer(self.h, ctypes.byref(desc),
                                                 None if epilogue is None else ctypes.byref(epilogue), handle))

    def int8_tile(self, product):
        """(rows, columns) of the tile that an Int8 or IntegerDesc runs on (gdy_integer_tile)."""
        d = product if isinstance(product, IntegerDesc) else product.descs()[0]
        rows, cols = ctypes.c_int32(), ctypes.c_int32()
        self._check(self.lib.gdy_integer_tile(self.h, ctypes.byref(d), ctypes.byref(rows), ctypes.byref(cols)))
        return rows.value, cols.value

    def set_rc(self, budget_cus: int):
        self._check(self.lib.gdy_set_rc(self.h, budget_cus))

    def set_timing(self, on: bool):
        self._check(self.lib.gdy_set_timing(self.h, int(on)))

    def kernel_times(self, n: int, back: int = 0):
        """(start_ms, end_ms) lists for the GEMMs of a timed submission
        (back = 0: the last one), relative to that submission's start."""
        s = (ctypes.c_float * max(n, 1))()
        e = (ctypes.c_float * max(n, 1))()
        self._check(self.lib.gdy_kernel_times(self.h, back, s, e, n))
        return list(s[:n]), list(e[:n])

    def dispatch_map(self, gemms, mode="selector", forced_cd: int = 0, dispatch: int = 0,
                     max_workgroups: int = 1 << 20) -> dict:
        """gdy_dispatch_map: per workgroup of one dispatch, the member it serves
        (-1: idle), its first work item and stride; per GEMM its item count."""
        arr = descs(gemms)
        n = len(gemms)
        grid = ctypes.c_int32()
        cap = max_workgroups
        gw = (ctypes.c_int32 * cap)()
        fi = (ctypes.c_int32 * cap)()
        st = (ctypes.c_int32 * cap)()
        items = (ctypes.c_int64 * max(n, 1))()
        self._check(self.lib.gdy_dispatch_map(self.h, arr, n, _mode(mode), forced_cd, dispatch, cap,
                                              ctypes.byref(grid), gw, fi, st, items))
        g = min(grid.value, cap)
        return {"grid": grid.value, "gemm": list(gw[:g]), "first": list(fi[:g]), "stride": list(st[:g]),
                "items": list(items[:n])}

    def features(self, gemm) -> list:
        d = gemm if isinstance(gemm, GemmDesc) else gemm.desc()
        out = (ctypes.c_double * N_FEATURES)()
        self._check(self.lib.gdy_features(self.h, ctypes.byref(d), out))
        return list(out)

    def variant_count(self) -> int:
        return int(self.lib.gdy_variant_count(self.h))

    def variant(self, vid: int) -> dict:
        v = VariantDesc()
        self._check(self.lib.gdy_variant_info(self.h, vid, ctypes.byref(v)))
        return v.as_dict()

    def variants(self) -> list:
        return [self.variant(i) for i in range(self.variant_count())]

    def find(self, name: str) -> int:
        return int(self.lib.gdy_variant_find(self.h, name.encode()))

    def isolated_variant(self, gemm) -> int:
        d = gemm if isinstance(gemm, GemmDesc) else gemm.desc()
        return int(self.lib.gdy_isolated_variant(self.h, ctypes.byref(d)))

    def catalogue_hash(self) -> int:
        return int(self.lib.gdy_catalogue_hash(self.h))

    def cus(self) -> int:
        return int(self.lib.gdy_device_cus(self.h))


def _mode(mode) -> int:
    return MODES[mode] if isinstance(mode, str) else int(mode)


def _stream_handle(stream, device=None):
    """None: torch's current stream of `device`, or of the current device."""
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)
    if hasattr(stream, "cuda_stream"):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))
