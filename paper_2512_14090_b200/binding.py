"""ctypes binding of libaiq.so: argument marshalling only.

Every function here has the name of the C entry point it calls (see include/aiq.h) and
does nothing but convert arguments: torch tensors supply device pointers and the current
stream, NumPy arrays supply host pointers.  All arithmetic runs inside the CUDA library;
if the library is missing the import of this module fails.
"""
import ctypes as C
import os

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libaiq.so")

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED_BITS, ERR_SHAPE, ERR_WORKSPACE_TOO_SMALL = 1, 2, 3, 4
ERR_CUDA, ERR_NOT_SM100, ERR_NONFINITE, ERR_TIMEOUT = 5, 6, 7, 8

LAYER_KIND = {"conv": 0, "dw": 1, "fc": 2}
ACT = {"none": 0, "relu": 1, "relu6": 2, "silu": 3, "gelu": 4, "gelu_tanh": 5}        # a model's layers take the first three
SCORE = {"softmax": 0, "sigmoid": 1}

EXPORTS = [
    "aiq_status_string", "aiq_last_error", "aiq_fold_bn", "aiq_packed_row_bytes",
    "aiq_quantize_layer", "aiq_qlinear", "aiq_qlinear_workspace_bytes", "aiq_model_bytes", "aiq_model_create",
    "aiq_model_destroy", "aiq_model_num_layers", "aiq_model_num_classes",
    "aiq_model_layer_folded", "aiq_model_layer_packed", "aiq_workspace_bytes", "aiq_forward",
    "aiq_eval_schemes", "aiq_set_eval_options", "aiq_set_fusion", "aiq_set_small_pass_images", "aiq_quantize_layer_per_tensor", "aiq_set_scale_granularity", "aiq_last_call_stats", "aiq_scheme_ai",
    "aiq_profile_start", "aiq_profile_stop", "aiq_forward_static",
    "aiq_mx_row_bytes", "aiq_mx_scale_row_bytes", "aiq_mx_quantize", "aiq_mx_dequantize", "aiq_mx_linear_workspace_bytes",
    "aiq_mx_linear", "aiq_mx_matmul", "aiq_debug_mx_expire_wait", "aiq_mx_linear_act",
    "aiq_expert_plan_bytes", "aiq_expert_plan_parts", "aiq_plan_experts", "aiq_route_experts", "aiq_mx_linear_experts_workspace_bytes",
    "aiq_mx_linear_experts", "aiq_combine_experts",
    "aiq_set_compute_path", "aiq_model_status", "aiq_debug_expire_wait", "aiq_search_greedy", "aiq_search_coordinate_descent",
]

PATH_AUTO, PATH_FP32, PATH_TENSOR, PATH_TENSOR_TILES = 0, 1, 2, 3

STATIC_WORKSPACE_BYTES = 8 * 1024 * 1024

KERNEL_KINDS = ["fold", "quantize", "qlinear", "conv", "depthwise", "pool", "argmax", "conv_tc"]


class AiqError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__(f"aiq status {status} ({status_string(status)}): {detail}")
        self.status = status


class LayerDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "cin", "cout", "ksize", "stride", "pad", "act",
                                         "input", "residual", "has_bn")]


class ArchDesc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("in_c", C.c_int32), ("in_h", C.c_int32),
                ("in_w", C.c_int32), ("layers", C.POINTER(LayerDesc))]


class KernelProfile(C.Structure):
    _fields_ = [("launches", C.c_int64), ("ms", C.c_double), ("flops", C.c_double),
                ("bytes", C.c_double)]


class SearchStep(C.Structure):
    _fields_ = [("layer", C.c_int32), ("bits", C.c_int32), ("accepted", C.c_int32), ("candidates", C.c_int32),
                ("loss", C.c_double), ("acc", C.c_double), ("ai", C.c_double)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("W", "gamma", "beta", "mean", "var", "bias")]


class _Int:
    """An `int` argument: out of its range, the smallest one, which every entry point refuses (c_int would keep the low 32 bits)."""

    @staticmethod
    def from_param(value):
        return C.c_int(value if -2 ** 31 <= value < 2 ** 31 else -2 ** 31)


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with "
                          "`python -m paper_2512_14090_b200.build` (there is no fallback path)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, f32, sz = C.c_void_p, C.c_int, C.c_float, C.c_size_t
    lib.aiq_status_string.restype = C.c_char_p
    lib.aiq_status_string.argtypes = [i32]
    lib.aiq_last_error.restype = C.c_char_p
    lib.aiq_last_error.argtypes = []
    lib.aiq_fold_bn.restype = i32
    lib.aiq_fold_bn.argtypes = [vp, vp, vp, vp, vp, i32, i32, f32, vp, vp, vp]
    lib.aiq_packed_row_bytes.restype = sz
    lib.aiq_packed_row_bytes.argtypes = [i32, i32]
    lib.aiq_quantize_layer.restype = i32
    lib.aiq_quantize_layer.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp]
    lib.aiq_qlinear.restype = i32
    lib.aiq_qlinear.argtypes = [vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, sz, vp]
    lib.aiq_qlinear_workspace_bytes.restype = sz
    lib.aiq_qlinear_workspace_bytes.argtypes = [i32, i32, i32, i32]
    i64, n32 = C.c_int64, _Int
    lib.aiq_mx_row_bytes.restype = sz
    lib.aiq_mx_row_bytes.argtypes = [n32]
    lib.aiq_mx_scale_row_bytes.restype = sz
    lib.aiq_mx_scale_row_bytes.argtypes = [n32]
    lib.aiq_mx_quantize.restype = i32
    lib.aiq_mx_quantize.argtypes = [vp, n32, n32, n32, i64, vp, vp, vp]
    lib.aiq_mx_dequantize.restype = i32
    lib.aiq_mx_dequantize.argtypes = [vp, vp, n32, n32, n32, vp, i64, vp]
    lib.aiq_mx_linear_workspace_bytes.restype = sz
    lib.aiq_mx_linear_workspace_bytes.argtypes = [n32, n32, n32, n32]
    lib.aiq_mx_linear.restype = i32
    lib.aiq_mx_linear.argtypes = [vp, vp, vp, n32, n32, vp, n32, n32, i64, vp, i64, vp, sz, vp]
    lib.aiq_mx_linear_act.restype = i32
    lib.aiq_mx_linear_act.argtypes = [vp, vp, vp, n32, n32, vp, n32, n32, i64, n32, n32, vp, i64, vp, i64, vp, sz, vp]
    lib.aiq_expert_plan_bytes.restype = sz
    lib.aiq_expert_plan_bytes.argtypes = [n32, n32, n32]
    lib.aiq_expert_plan_parts.restype = i32
    lib.aiq_expert_plan_parts.argtypes = [n32, n32, n32, C.POINTER(sz), C.POINTER(sz), C.POINTER(sz)]
    lib.aiq_plan_experts.restype = i32
    lib.aiq_plan_experts.argtypes = [vp, n32, n32, n32, vp, sz, vp]
    lib.aiq_route_experts.restype = i32
    lib.aiq_route_experts.argtypes = [vp, n32, n32, n32, i64, vp, n32, n32, n32, n32, n32, n32, f32, vp, vp, vp, sz, vp]
    lib.aiq_mx_linear_experts_workspace_bytes.restype = sz
    lib.aiq_mx_linear_experts_workspace_bytes.argtypes = [n32, n32, n32, n32, n32]
    lib.aiq_mx_linear_experts.restype = i32
    lib.aiq_mx_linear_experts.argtypes = [vp, vp, vp, n32, n32, n32, vp, n32, i64, n32, vp, sz, n32, n32, n32, n32, vp, i64, vp, sz, vp]
    lib.aiq_combine_experts.restype = i32
    lib.aiq_combine_experts.argtypes = [vp, n32, n32, n32, n32, n32, i64, vp, vp, sz, vp, i64, vp, i64, vp]
    lib.aiq_debug_mx_expire_wait.restype = i32
    lib.aiq_debug_mx_expire_wait.argtypes = [i64]
    lib.aiq_mx_matmul.restype = i32
    lib.aiq_mx_matmul.argtypes = [vp, vp, n32, vp, vp, n32, vp, n32, vp, n32, i64, vp]
    lib.aiq_model_bytes.restype = sz
    lib.aiq_model_bytes.argtypes = [C.POINTER(ArchDesc)]
    lib.aiq_model_create.restype = i32
    lib.aiq_model_create.argtypes = [C.POINTER(ArchDesc), C.POINTER(LayerWeights), vp, sz, vp,
                                     C.POINTER(vp)]
    lib.aiq_model_destroy.restype = None
    lib.aiq_model_destroy.argtypes = [vp]
    lib.aiq_model_num_layers.restype = i32
    lib.aiq_model_num_layers.argtypes = [vp]
    lib.aiq_model_num_classes.restype = i32
    lib.aiq_model_num_classes.argtypes = [vp]
    lib.aiq_model_layer_folded.restype = i32
    lib.aiq_model_layer_folded.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(i32),
                                           C.POINTER(i32)]
    lib.aiq_model_layer_packed.restype = i32
    lib.aiq_model_layer_packed.argtypes = [vp, i32, i32, C.POINTER(vp), C.POINTER(vp)]
    lib.aiq_workspace_bytes.restype = sz
    lib.aiq_workspace_bytes.argtypes = [vp, i32, i32]
    lib.aiq_forward.restype = i32
    lib.aiq_forward.argtypes = [vp, vp, vp, i32, vp, vp, sz, vp]
    lib.aiq_eval_schemes.restype = i32
    lib.aiq_eval_schemes.argtypes = [vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.aiq_set_eval_options.restype = None
    lib.aiq_set_eval_options.argtypes = [i32, i32]
    lib.aiq_quantize_layer_per_tensor.restype = i32
    lib.aiq_quantize_layer_per_tensor.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.aiq_set_scale_granularity.restype = None
    lib.aiq_set_scale_granularity.argtypes = [i32]
    lib.aiq_set_fusion.restype = None
    lib.aiq_set_fusion.argtypes = [i32, i32]
    lib.aiq_set_small_pass_images.restype = None
    lib.aiq_set_small_pass_images.argtypes = [i32]
    lib.aiq_last_call_stats.restype = None
    lib.aiq_last_call_stats.argtypes = [C.POINTER(C.c_int64)] * 3
    lib.aiq_search_greedy.restype = i32
    lib.aiq_search_greedy.argtypes = [vp, vp, i32, vp, i32, C.c_double, vp, vp, i32, vp,
                                      C.POINTER(SearchStep), i32, C.POINTER(C.c_int), vp, sz, vp]
    lib.aiq_search_coordinate_descent.restype = i32
    lib.aiq_search_coordinate_descent.argtypes = [vp, vp, i32, vp, i32, C.c_double, i32, vp, vp, i32, vp,
                                                  C.POINTER(SearchStep), i32, C.POINTER(C.c_int), vp, sz, vp]
    lib.aiq_scheme_ai.restype = i32
    lib.aiq_scheme_ai.argtypes = [vp, vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                  C.POINTER(C.c_double)]
    lib.aiq_forward_static.restype = i32
    lib.aiq_forward_static.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.aiq_model_status.restype = i32
    lib.aiq_model_status.argtypes = [vp, vp]
    lib.aiq_debug_expire_wait.restype = i32
    lib.aiq_debug_expire_wait.argtypes = [vp, C.c_int64, vp]
    lib.aiq_set_compute_path.restype = None
    lib.aiq_set_compute_path.argtypes = [i32]
    lib.aiq_profile_start.restype = i32
    lib.aiq_profile_start.argtypes = []
    lib.aiq_profile_stop.restype = i32
    lib.aiq_profile_stop.argtypes = [C.POINTER(KernelProfile)]
    return lib


lib = _load()


def status_string(status):
    return lib.aiq_status_string(int(status)).decode()


def last_error():
    return lib.aiq_last_error().decode()


def _check(status):
    if status != OK:
        raise AiqError(status, last_error())


# A small call spends more time here than on the GPU (MobileNetV2's classifier-sized linear layer, one row: 10.0 us a
# call with a c_void_p object per argument and torch.cuda.current_stream(), 5.3 us with plain integers and the raw
# stream handle), so pointers are passed as integers; the argument types of the library convert them.
def _dev(t):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return t.data_ptr()


def _host(a):
    return a.__array_interface__["data"][0] if a is not None else None


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()                     # initialises CUDA
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # not a public name: the public call where it is gone
        _raw_stream = (torch.cuda.current_device, raw or (lambda device: torch.cuda.current_stream(device).cuda_stream))
    device, raw = _raw_stream
    return raw(device())


_raw_stream = None


def arch_desc(arch):
    """(ArchDesc, keep-alive list) from an architecture dict (kind/cin/cout/k/...)."""
    layers = (LayerDesc * len(arch["layers"]))()
    for d, l in zip(layers, arch["layers"]):
        d.kind, d.cin, d.cout, d.ksize = LAYER_KIND[l["kind"]], l["cin"], l["cout"], l["k"]
        d.stride, d.pad, d.act = l["stride"], l["pad"], ACT[l["act"]]
        d.input, d.residual, d.has_bn = l["input"], l["residual"], int(bool(l["has_bn"]))
    desc = ArchDesc(len(arch["layers"]), arch["in_c"], arch["in_h"], arch["in_w"], layers)
    return desc, layers


# ------------------------------------------------------------------------- plain calls
def aiq_packed_row_bytes(K, bits):
    return int(lib.aiq_packed_row_bytes(int(K), int(bits)))


def aiq_fold_bn(W, gamma, beta, mean, var, Wf, bf, eps=1e-5, stream=None):
    N = W.shape[0]
    K = W.numel() // N
    _check(lib.aiq_fold_bn(_dev(W), _dev(gamma), _dev(beta), _dev(mean), _dev(var), N, K,
                           C.c_float(eps), _dev(Wf), _dev(bf), _stream(stream)))


def aiq_quantize_layer(W, bits, packed_out, scales_out, nonfinite_flag=None, stream=None):
    N, K = W.shape
    _check(lib.aiq_quantize_layer(_dev(W), N, K, int(bits), _dev(packed_out), _dev(scales_out),
                                  _dev(nonfinite_flag), _stream(stream)))


def aiq_qlinear_workspace_bytes(N, K, bits, M):
    return int(lib.aiq_qlinear_workspace_bytes(int(N), int(K), int(bits), int(M)))


def aiq_qlinear(packed, scales, bias, N, K, bits, x, y, workspace=None, stream=None):
    status = lib.aiq_qlinear(_dev(packed), _dev(scales), _dev(bias), int(N), int(K), int(bits), _dev(x), x.shape[0], _dev(y),
                             _dev(workspace), workspace.numel() if workspace is not None else 0, _stream(stream))
    if status:
        _check(status)


# ------------------------------------------------------------------- microscaled 4 bits
DTYPE_F32, DTYPE_F16, DTYPE_BF16 = 0, 1, 2

# These calls take their arguments through a CPython module (csrc/mxcall.c) where it is built, else through ctypes.
try:
    from . import _mxcall
except ImportError:
    _mxcall = lib
_dtypes = None


def _dtype(dtype):
    """AIQ_DTYPE_* of a torch type (or of itself)."""
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = {torch.float32: DTYPE_F32, torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16,
                   DTYPE_F32: DTYPE_F32, DTYPE_F16: DTYPE_F16, DTYPE_BF16: DTYPE_BF16}
    code = _dtypes.get(dtype)
    if code is None:
        raise ValueError(f"expected float32, float16 or bfloat16, not {dtype}")
    return code


# Shapes, strides and types decide all that the checks below look at; their answers are kept for the next call with the same ones
# (a check takes as long as a kernel launch).  What else can differ is looked at every time.
def _mx_plan(key, check, *args):
    plan = check(*args)
    if len(_mx_plans) >= 4096:
        _mx_plans.clear()
    _mx_plans[key] = plan
    return plan


_mx_plans = {}


def _mx_stream(stream, device, same):
    """The launch goes to the current device (its current stream): `device`, where `same` says that every tensor lies."""
    if _raw_stream is None:
        _stream()
    current, raw = _raw_stream
    if not same or device != current():                     # -1: not a CUDA tensor
        raise ValueError(f"expected every tensor on the current device, cuda:{current()}")
    return raw(device) if stream is None else stream.cuda_stream


def _mx_rows(t):
    """(type, rows, K, row stride) of a matrix whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError(f"expected a matrix, not {tuple(t.shape)}")
    rows, k = t.shape
    stride, step = t.stride()
    if step != 1 and k != 1:
        raise ValueError("expected contiguous rows")
    return _dtype(t.dtype), rows, k, stride


def _mx_held(codes, scales, k):
    """The rows of k values each that codes and scales hold."""
    if not codes.is_cuda or not scales.is_cuda:
        raise ValueError("expected CUDA tensors")
    if codes.dim() != 2:
        raise ValueError(f"expected codes of bytes, a row per row of values, not {tuple(codes.shape)}")
    rows = codes.shape[0]
    want = (rows, (k + 127) // 128 * 64), (rows, (k + 511) // 512 * 16)
    if (tuple(codes.shape), tuple(scales.shape)) != want or codes.element_size() != 1 or scales.element_size() != 1:
        raise ValueError(f"expected codes and scales of bytes, {want[0]} and {want[1]} for rows of {k} values, not {tuple(codes.shape)} and "
                         f"{tuple(scales.shape)}")
    if not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("expected contiguous codes and scales")
    return rows


def _mx_bias(bias, n):
    if bias is not None and (bias.numel() != n or bias.element_size() != 4 or not bias.is_floating_point() or not bias.is_contiguous()):
        raise ValueError(f"expected a contiguous float32 bias of {n} values")


def _mx_check_values(codes, scales, values):
    dtype, rows, k, stride = _mx_rows(values)
    if _mx_held(codes, scales, k) != rows:
        raise ValueError(f"codes of {codes.shape[0]} rows and {rows} rows of values")
    return dtype, rows, k, stride


def _mx_check_linear(codes, scales, bias, x, y):
    dtype, m, k, x_stride = _mx_rows(x)
    y_dtype, y_rows, n, y_stride = _mx_rows(y)
    held = _mx_held(codes, scales, k)
    if (y_dtype, y_rows, held) != (dtype, m, n):
        raise ValueError(f"x {tuple(x.shape)} {x.dtype}, weights of {held} rows and y {tuple(y.shape)} {y.dtype} do not match")
    _mx_bias(bias, n)
    return n, k, dtype, m, x_stride, y_stride


def _mx_check_matmul(a_codes, a_scales, b_codes, b_scales, bias, y, K):
    dtype, m, n, y_stride = _mx_rows(y)
    rows = _mx_held(a_codes, a_scales, K), _mx_held(b_codes, b_scales, K)
    if rows != (m, n):
        raise ValueError(f"A of {rows[0]} rows, B of {rows[1]} and y {tuple(y.shape)} do not match")
    _mx_bias(bias, n)
    return m, n, dtype, y_stride


def _choice(names, name, what):
    code = names.get(name)
    if code is None:
        raise ValueError(f"expected one of {', '.join(names)} as {what}, not {name!r}")
    return code


def _mx_outputs(n, gated):
    if gated and n % 2:
        raise ValueError(f"gated, but weights of {n} rows")
    return n // 2 if gated else n


def _mx_check_linear_act(codes, scales, bias, x, y, activation, gated, residual):
    act = _choice(ACT, activation, "activation")
    dtype, m, k, x_stride = _mx_rows(x)
    y_dtype, y_rows, outputs, y_stride = _mx_rows(y)
    n = _mx_held(codes, scales, k)
    if (y_dtype, y_rows, outputs) != (dtype, m, _mx_outputs(n, gated)):
        raise ValueError(f"x {tuple(x.shape)} {x.dtype}, weights of {n} rows and y {tuple(y.shape)} {y.dtype} do not match")
    _mx_bias(bias, n)
    r_stride = 0
    if residual is not None:
        r_dtype, r_rows, r_width, r_stride = _mx_rows(residual)
        if (r_dtype, r_rows, r_width) != (dtype, m, outputs):
            raise ValueError(f"residual {tuple(residual.shape)} {residual.dtype} and y {tuple(y.shape)} {y.dtype} do not match")
    return n, k, dtype, m, x_stride, act, int(bool(gated)), r_stride, y_stride


def _expert_array(t, dtype, shape, what):
    if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"expected {what} as a contiguous {dtype} {shape}, not {t.dtype} {tuple(t.shape)}")


def _expert_plan(plan, T, top_k, E):
    """Bytes of a plan that is large enough."""
    needed = int(lib.aiq_expert_plan_bytes(T, top_k, E))
    if needed == 0:
        _check(lib.aiq_expert_plan_parts(T, top_k, E, None, None, None))
    size = plan.numel() * plan.element_size()
    if not plan.is_contiguous() or size < needed:
        raise ValueError(f"expected a contiguous plan of {needed} bytes for {T} tokens, {top_k} of {E} experts, not {size}")
    return size


def _check_route(logits, ids, weights, bias, scoring, plan):
    import torch
    dtype, t, e, stride = _mx_rows(logits)
    if ids.dim() != 2:
        raise ValueError(f"expected ids of a row per token, not {tuple(ids.shape)}")
    top_k = ids.shape[1]
    _expert_array(ids, torch.int32, (t, top_k), "ids")
    _expert_array(weights, torch.float32, (t, top_k), "weights")
    _mx_bias(bias, e)
    return dtype, t, e, stride, _choice(SCORE, scoring, "scoring"), top_k, 0 if plan is None else _expert_plan(plan, t, top_k, e)


def _check_plan(ids, plan, e):
    import torch
    if ids.dim() != 2:
        raise ValueError(f"expected ids of a row per token, not {tuple(ids.shape)}")
    t, top_k = ids.shape
    _expert_array(ids, torch.int32, (t, top_k), "ids")
    return t, top_k, _expert_plan(plan, t, top_k, e)


def _check_experts(codes, scales, bias, x, plan, top_k, y, activation, gated, x_sorted):
    act = _choice(ACT, activation, "activation")
    dtype, x_rows, k, x_stride = _mx_rows(x)
    y_dtype, rows, outputs, y_stride = _mx_rows(y)
    if codes.dim() != 3 or scales.dim() != 3:
        raise ValueError(f"expected codes and scales of a matrix per expert, not {tuple(codes.shape)} and {tuple(scales.shape)}")
    e, n = codes.shape[:2]
    if scales.shape[0] != e or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("expected contiguous codes and scales of as many experts")
    _mx_held(codes.reshape(e * n, codes.shape[2]), scales.reshape(e * scales.shape[1], scales.shape[2]), k)
    t = rows // top_k if top_k > 0 else 0
    if (y_dtype, t * top_k, outputs) != (dtype, rows, _mx_outputs(n, gated)) or x_rows != (rows if x_sorted else t):
        raise ValueError(f"x {tuple(x.shape)} {x.dtype}, {top_k} of {e} experts of {n} rows and y {tuple(y.shape)} {y.dtype} do not match")
    if bias is not None and tuple(bias.shape) != (e, n):
        raise ValueError(f"expected a bias of {(e, n)}, not {tuple(bias.shape)}")
    _mx_bias(bias, e * n)
    return e, n, k, dtype, x_stride, int(bool(x_sorted)), _expert_plan(plan, t, top_k, e), t, act, int(bool(gated)), y_stride


def _check_combine(z, weights, plan, e, y, residual):
    import torch
    dtype, rows, width, z_stride = _mx_rows(z)
    if weights.dim() != 2:
        raise ValueError(f"expected weights of a row per token, not {tuple(weights.shape)}")
    t, top_k = weights.shape
    _expert_array(weights, torch.float32, (t, top_k), "weights")
    r_stride = 0
    for what, m, of in (("z", z, t * top_k), ("y", y, t), ("residual", residual, t)):
        if m is not None:
            m_dtype, m_rows, m_width, stride = _mx_rows(m)
            if (m_dtype, m_rows, m_width) != (dtype, of, width):
                raise ValueError(f"{what} {tuple(m.shape)} {m.dtype}, z {tuple(z.shape)} {z.dtype} and weights {(t, top_k)} do not match")
            if what == "y":
                y_stride = stride
            elif what == "residual":
                r_stride = stride
    return dtype, t, top_k, width, z_stride, _expert_plan(plan, t, top_k, e), r_stride, y_stride


def aiq_mx_row_bytes(K):
    return int(lib.aiq_mx_row_bytes(int(K)))


def aiq_mx_scale_row_bytes(K):
    return int(lib.aiq_mx_scale_row_bytes(int(K)))


def aiq_mx_quantize(x, codes_out, scales_out, stream=None):
    """x [rows][K] float32, float16 or bfloat16 (rows may have any stride) -> codes_out uint8 [rows][aiq_mx_row_bytes(K)],
    scales_out uint8 [rows][aiq_mx_scale_row_bytes(K)]."""
    key = (codes_out.shape, scales_out.shape, x.shape, x.stride(), x.dtype, codes_out.dtype, scales_out.dtype,
           codes_out.is_contiguous(), scales_out.is_contiguous())
    dtype, rows, k, stride = _mx_plans.get(key) or _mx_plan(key, _mx_check_values, codes_out, scales_out, x)
    d = x.get_device()
    s = _mx_stream(stream, d, d == codes_out.get_device() == scales_out.get_device())
    status = _mxcall.aiq_mx_quantize(x.data_ptr(), dtype, rows, k, stride, codes_out.data_ptr(), scales_out.data_ptr(), s)
    if status:
        _check(status)


def aiq_mx_dequantize(codes, scales, y, stream=None):
    """codes, scales -> y [rows][K] float32, float16 or bfloat16."""
    key = (codes.shape, scales.shape, y.shape, y.stride(), y.dtype, codes.dtype, scales.dtype, codes.is_contiguous(), scales.is_contiguous())
    dtype, rows, k, stride = _mx_plans.get(key) or _mx_plan(key, _mx_check_values, codes, scales, y)
    d = y.get_device()
    s = _mx_stream(stream, d, d == codes.get_device() == scales.get_device())
    status = _mxcall.aiq_mx_dequantize(codes.data_ptr(), scales.data_ptr(), rows, k, dtype, y.data_ptr(), stride, s)
    if status:
        _check(status)


def aiq_mx_linear_workspace_bytes(N, K, M, dtype):
    return int(lib.aiq_mx_linear_workspace_bytes(int(N), int(K), int(M), _dtype(dtype)))


def aiq_mx_linear(codes, scales, bias, x, y, workspace=None, stream=None):
    """y [M][N] = x [M][K] * W^T + bias; W [N][K] as codes and scales, x and y of one type, bias float32 [N] or None.  workspace: a tensor of
    aiq_mx_linear_workspace_bytes(N, K, M, x.dtype) bytes; without one large products leave the tensor cores and take up to 100 times as long."""
    key = (codes.shape, scales.shape, x.shape, y.shape, x.stride(), y.stride(), x.dtype, y.dtype, codes.dtype, scales.dtype,
           codes.is_contiguous(), scales.is_contiguous(), (bias.shape, bias.dtype, bias.is_contiguous()) if bias is not None else None)
    n, k, dtype, m, x_stride, y_stride = _mx_plans.get(key) or _mx_plan(key, _mx_check_linear, codes, scales, bias, x, y)
    d = x.get_device()
    s = _mx_stream(stream, d, d == y.get_device() == codes.get_device() == scales.get_device()
                   and (bias is None or bias.get_device() == d) and (workspace is None or workspace.get_device() == d))
    ws, size = (_dev(workspace), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    status = _mxcall.aiq_mx_linear(codes.data_ptr(), scales.data_ptr(), bias.data_ptr() if bias is not None else None, n, k, x.data_ptr(), dtype,
                               m, x_stride, y.data_ptr(), y_stride, ws, size, s)
    if status:
        _check(status)


def aiq_mx_matmul(a_codes, a_scales, b_codes, b_scales, bias, K, y, stream=None):
    """y [M][N] = A [M][K] * B [N][K]^T + bias; both matrices as codes and scales, y float32, float16 or bfloat16."""
    key = (K, a_codes.shape, a_scales.shape, b_codes.shape, b_scales.shape, y.shape, y.stride(), y.dtype, a_codes.dtype, a_scales.dtype,
           b_codes.dtype, b_scales.dtype, a_codes.is_contiguous(), a_scales.is_contiguous(), b_codes.is_contiguous(),
           b_scales.is_contiguous(), (bias.shape, bias.dtype, bias.is_contiguous()) if bias is not None else None)
    m, n, dtype, y_stride = _mx_plans.get(key) or _mx_plan(key, _mx_check_matmul, a_codes, a_scales, b_codes, b_scales, bias, y, int(K))
    d = y.get_device()
    s = _mx_stream(stream, d, d == a_codes.get_device() == a_scales.get_device() == b_codes.get_device() == b_scales.get_device()
                   and (bias is None or bias.get_device() == d))
    status = _mxcall.aiq_mx_matmul(a_codes.data_ptr(), a_scales.data_ptr(), m, b_codes.data_ptr(), b_scales.data_ptr(), n,
                               bias.data_ptr() if bias is not None else None, int(K), y.data_ptr(), dtype, y_stride, s)
    if status:
        _check(status)


def aiq_mx_linear_act(codes, scales, bias, x, y, activation="none", gated=False, residual=None, workspace=None, stream=None):
    """y [M][N] = act(x W^T + bias) + residual; gated: y [M][N / 2] = act(x G^T + bias_g) * (x U^T + bias_u) + residual, G and U the first and the second
    half of the rows of W.  activation: "none", "relu", "relu6", "silu", "gelu" or "gelu_tanh"; residual as y, which it may be.  The rest as
    aiq_mx_linear, the workspace's size too."""
    key = (activation, gated, codes.shape, scales.shape, x.shape, y.shape, x.stride(), y.stride(), x.dtype, y.dtype, codes.dtype, scales.dtype,
           codes.is_contiguous(), scales.is_contiguous(), (bias.shape, bias.dtype, bias.is_contiguous()) if bias is not None else None,
           (residual.shape, residual.stride(), residual.dtype) if residual is not None else None)
    n, k, dtype, m, x_stride, act, gate, r_stride, y_stride = (
        _mx_plans.get(key) or _mx_plan(key, _mx_check_linear_act, codes, scales, bias, x, y, activation, gated, residual))
    d = x.get_device()
    s = _mx_stream(stream, d, d == y.get_device() == codes.get_device() == scales.get_device()
                   and (bias is None or bias.get_device() == d) and (residual is None or residual.get_device() == d)
                   and (workspace is None or workspace.get_device() == d))
    ws, size = (_dev(workspace), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    status = _mxcall.aiq_mx_linear_act(codes.data_ptr(), scales.data_ptr(), bias.data_ptr() if bias is not None else None, n, k, x.data_ptr(), dtype, m,
                                       x_stride, act, gate, residual.data_ptr() if residual is not None else None, r_stride, y.data_ptr(), y_stride,
                                       ws, size, s)
    if status:
        _check(status)


# ------------------------------------------------------------------------------- experts
def aiq_expert_plan_bytes(T, top_k, E):
    return int(lib.aiq_expert_plan_bytes(int(T), int(top_k), int(E)))


def aiq_expert_plan_parts(plan, T, top_k, E):
    """Views of a plan's int32 parts: offsets [E + 1], slots [T * top_k], positions [T][top_k]."""
    key = ("parts", T, top_k, E)
    at = _mx_plans.get(key)
    if at is None:
        starts = [C.c_size_t() for _ in range(3)]
        _check(lib.aiq_expert_plan_parts(T, top_k, E, *[C.byref(a) for a in starts]))
        at = _mx_plans[key] = [a.value // 4 for a in starts]
    import torch
    w = plan.view(torch.int32)
    return (w.as_strided((E + 1,), (1,), w.storage_offset() + at[0]), w.as_strided((T * top_k,), (1,), w.storage_offset() + at[1]),
            w.as_strided((T, top_k), (top_k, 1), w.storage_offset() + at[2]))


def aiq_plan_experts(ids, E, plan, stream=None):
    """ids int32 [T][top_k] -> plan, a tensor of aiq_expert_plan_bytes(T, top_k, E) bytes."""
    key = (E, ids.shape, ids.dtype, ids.is_contiguous(), plan.shape, plan.dtype, plan.is_contiguous())
    t, top_k, size = _mx_plans.get(key) or _mx_plan(key, _check_plan, ids, plan, int(E))
    d = ids.get_device()
    s = _mx_stream(stream, d, d == plan.get_device())
    status = _mxcall.aiq_plan_experts(ids.data_ptr(), t, top_k, int(E), plan.data_ptr(), size, s)
    if status:
        _check(status)


def aiq_route_experts(logits, ids, weights, bias=None, scoring="softmax", groups=1, top_groups=1, group_best=1, renormalise=True, scale=1.0, plan=None,
                      stream=None):
    """logits [T][E] float32, float16 or bfloat16 -> ids int32 [T][top_k], weights float32 [T][top_k] and, where given, a plan of
    aiq_expert_plan_bytes(T, top_k, E) bytes.  scoring: "softmax" or "sigmoid"; bias float32 [E] or None."""
    key = (scoring, logits.shape, logits.stride(), logits.dtype, ids.shape, ids.dtype, ids.is_contiguous(), weights.shape, weights.dtype,
           weights.is_contiguous(), (bias.shape, bias.dtype, bias.is_contiguous()) if bias is not None else None,
           (plan.shape, plan.dtype, plan.is_contiguous()) if plan is not None else None)
    dtype, t, e, stride, score, top_k, size = _mx_plans.get(key) or _mx_plan(key, _check_route, logits, ids, weights, bias, scoring, plan)
    d = logits.get_device()
    s = _mx_stream(stream, d, d == ids.get_device() == weights.get_device() and (bias is None or bias.get_device() == d)
                   and (plan is None or plan.get_device() == d))
    status = _mxcall.aiq_route_experts(logits.data_ptr(), dtype, t, e, stride, bias.data_ptr() if bias is not None else None, score, top_k,
                                       int(groups), int(top_groups), int(group_best), int(bool(renormalise)), float(scale), ids.data_ptr(),
                                       weights.data_ptr(), plan.data_ptr() if plan is not None else None, size, s)
    if status:
        _check(status)


def aiq_mx_linear_experts_workspace_bytes(E, N, K, rows, dtype):
    return int(lib.aiq_mx_linear_experts_workspace_bytes(int(E), int(N), int(K), int(rows), _dtype(dtype)))


def aiq_mx_linear_experts(codes, scales, bias, x, plan, top_k, y, activation="none", gated=False, x_sorted=False, workspace=None, stream=None):
    """y [T * top_k][N, gated: N / 2] = act(x W^T + bias) for the plan's rows, with each row's expert's weights: codes [E][N][aiq_mx_row_bytes(K)], scales
    [E][N][aiq_mx_scale_row_bytes(K)], bias float32 [E][N] or None.  x [T][K], or [T * top_k][K] in the plan's rows (x_sorted).  workspace: a tensor of
    aiq_mx_linear_experts_workspace_bytes(E, N, K, T * top_k, x.dtype) bytes."""
    key = (activation, gated, x_sorted, top_k, codes.shape, codes.dtype, codes.is_contiguous(), scales.shape, scales.dtype, scales.is_contiguous(),
           (bias.shape, bias.dtype, bias.is_contiguous()) if bias is not None else None, x.shape, x.stride(), x.dtype, y.shape, y.stride(), y.dtype,
           plan.shape, plan.dtype, plan.is_contiguous())
    e, n, k, dtype, x_stride, in_order, size, t, act, gate, y_stride = (
        _mx_plans.get(key) or _mx_plan(key, _check_experts, codes, scales, bias, x, plan, int(top_k), y, activation, gated, x_sorted))
    if workspace is None:
        raise ValueError("expected a workspace")
    d = x.get_device()
    s = _mx_stream(stream, d, d == y.get_device() == codes.get_device() == scales.get_device() == plan.get_device() == workspace.get_device()
                   and (bias is None or bias.get_device() == d))
    status = _mxcall.aiq_mx_linear_experts(codes.data_ptr(), scales.data_ptr(), bias.data_ptr() if bias is not None else None, e, n, k, x.data_ptr(), dtype,
                                           x_stride, in_order, plan.data_ptr(), size, t, int(top_k), act, gate, y.data_ptr(), y_stride,
                                           _dev(workspace), workspace.numel() * workspace.element_size(), s)
    if status:
        _check(status)


def aiq_combine_experts(z, weights, plan, E, y, residual=None, stream=None):
    """y [T][H] = residual + the weighted sum of each token's rows of z [T * top_k][H]; weights float32 [T][top_k]; residual as y, which it may be."""
    key = (E, z.shape, z.stride(), z.dtype, weights.shape, weights.dtype, weights.is_contiguous(), plan.shape, plan.dtype, plan.is_contiguous(),
           y.shape, y.stride(), y.dtype, (residual.shape, residual.stride(), residual.dtype) if residual is not None else None)
    dtype, t, top_k, width, z_stride, size, r_stride, y_stride = (
        _mx_plans.get(key) or _mx_plan(key, _check_combine, z, weights, plan, int(E), y, residual))
    d = z.get_device()
    s = _mx_stream(stream, d, d == weights.get_device() == plan.get_device() == y.get_device() and (residual is None or residual.get_device() == d))
    status = _mxcall.aiq_combine_experts(z.data_ptr(), dtype, t, top_k, int(E), width, z_stride, weights.data_ptr(), plan.data_ptr(), size,
                                         residual.data_ptr() if residual is not None else None, r_stride, y.data_ptr(), y_stride, s)
    if status:
        _check(status)


def aiq_debug_mx_expire_wait(limit_cycles):
    _check(lib.aiq_debug_mx_expire_wait(int(limit_cycles)))


def aiq_set_eval_options(chunk=0, share_prefix=True):
    lib.aiq_set_eval_options(int(chunk), int(bool(share_prefix)))


SCALE_PER_CHANNEL, SCALE_PER_TENSOR = 0, 1


def aiq_set_scale_granularity(granularity):
    lib.aiq_set_scale_granularity(int(granularity))


def aiq_quantize_layer_per_tensor(W, bits, packed_out, scales_out, scratch, nonfinite_flag=None, stream=None):
    N, K = W.shape
    _check(lib.aiq_quantize_layer_per_tensor(_dev(W), int(N), int(K), int(bits), _dev(packed_out), _dev(scales_out),
                                             _dev(nonfinite_flag), _dev(scratch), _stream(stream)))


def aiq_set_fusion(blocks=True, pool=True, inverted_residual="auto"):
    """inverted_residual: True (every eligible block), False, or "auto" (where the fused kernel is faster whatever the
    batch: at present no block)."""
    ir = 4 if inverted_residual == "auto" else (2 if inverted_residual else 0)
    lib.aiq_set_fusion(int(bool(blocks)) | ir, int(bool(pool)))


def aiq_set_small_pass_images(image_schemes):
    lib.aiq_set_small_pass_images(int(image_schemes))


def aiq_set_compute_path(path):
    lib.aiq_set_compute_path(int(path))


def aiq_last_call_stats():
    a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
    lib.aiq_last_call_stats(C.byref(a), C.byref(b), C.byref(c))
    return dict(kernel_launches=a.value, layer_evals=b.value, layer_evals_unshared=c.value)


def aiq_profile_start():
    _check(lib.aiq_profile_start())


def aiq_profile_stop():
    """{kind: dict(launches, ms, flops, bytes)} for the launches since aiq_profile_start."""
    out = (KernelProfile * len(KERNEL_KINDS))()
    _check(lib.aiq_profile_stop(out))
    return {k: dict(launches=o.launches, ms=o.ms, flops=o.flops, bytes=o.bytes)
            for k, o in zip(KERNEL_KINDS, out)}


# ------------------------------------------------------------------------- model object
class Model:
    """Owns the device memory the C model lives in (a torch uint8 tensor) and the handle."""

    def __init__(self, arch, params, device="cuda:0", stream=None, mem=None):
        """Uploads `params` (host float32 arrays), folds and builds the weight bank.
        `mem`: an existing uint8 CUDA tensor to build into (reused across rebuilds)."""
        import torch
        self.arch = arch
        self.device = torch.device(device)
        desc, self._keep_layers = arch_desc(arch)
        self._desc = desc
        nbytes = int(lib.aiq_model_bytes(C.byref(desc)))
        if nbytes == 0:
            raise AiqError(ERR_INVALID_ARG, last_error())
        if mem is not None and mem.numel() >= nbytes:
            self.mem = mem
        else:
            self.mem = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        weights = (LayerWeights * len(params))()
        keep = []
        for w, p in zip(weights, params):
            for name in ("W", "gamma", "beta", "mean", "var", "bias"):
                if name in p and p[name] is not None:
                    a = np.ascontiguousarray(p[name], dtype=np.float32)
                    keep.append(a)
                    setattr(w, name, a.__array_interface__["data"][0])
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib.aiq_model_create(C.byref(desc), weights, _dev(self.mem), self.mem.numel(),
                                        _stream(stream), C.byref(handle)))
        self.handle = handle
        self.n_layers = int(lib.aiq_model_num_layers(handle))
        self.n_classes = int(lib.aiq_model_num_classes(handle))
        self._ws = None

    def close(self):
        if getattr(self, "handle", None) and lib is not None:      # lib is None at interpreter exit
            lib.aiq_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()

    # views for inspection --------------------------------------------------------
    def layer_folded(self, layer):
        """(Wf [N][K], bias [N]) as torch views into the model memory."""
        wf, b, n, k = C.c_void_p(), C.c_void_p(), C.c_int(), C.c_int()
        _check(lib.aiq_model_layer_folded(self.handle, layer, C.byref(wf), C.byref(b), C.byref(n), C.byref(k)))
        return (self._view(wf.value, n.value * k.value * 4).view(dtype=_f32()).view(n.value, k.value),
                self._view(b.value, n.value * 4).view(dtype=_f32()))

    def layer_packed(self, layer, bits):
        p, s = C.c_void_p(), C.c_void_p()
        _check(lib.aiq_model_layer_packed(self.handle, layer, int(bits), C.byref(p), C.byref(s)))
        l = self._keep_layers[layer]                    # as the library was given it: the caller's dict may have changed
        n, k = l.cout, l.cin if l.kind == LAYER_KIND["fc"] else (1 if l.kind == LAYER_KIND["dw"] else l.cin) * l.ksize * l.ksize
        rb = aiq_packed_row_bytes(k, bits)
        return (self._view(p.value, n * rb).view(n, rb), self._view(s.value, n * 4).view(dtype=_f32()))

    def _view(self, ptr, nbytes):
        off = ptr - self.mem.data_ptr()
        assert 0 <= off and off + nbytes <= self.mem.numel()
        return self.mem[off:off + nbytes]

    # workspace -------------------------------------------------------------------
    def aiq_workspace_bytes(self, max_batch, max_schemes):
        return int(lib.aiq_workspace_bytes(self.handle, int(max_batch), int(max_schemes)))

    def workspace(self, max_batch, max_schemes):
        import torch
        need = self.aiq_workspace_bytes(max_batch, max_schemes)
        if self._ws is None or self._ws.numel() < need:
            self._ws = None
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    # the calls -------------------------------------------------------------------
    def aiq_forward(self, scheme_bits, x, logits=None, workspace=None, stream=None):
        import torch
        scheme = np.ascontiguousarray(scheme_bits, dtype=np.uint8)
        if scheme.shape != (self.n_layers,):
            raise ValueError("scheme length must equal the number of layers")
        B = x.shape[0]
        if logits is None:
            logits = torch.empty((B, self.n_classes), dtype=torch.float32, device=self.device)
        ws = workspace if workspace is not None else self.workspace(B, 1)
        _check(lib.aiq_forward(self.handle, _host(scheme), _dev(x), B, _dev(logits), _dev(ws),
                               ws.numel(), _stream(stream)))
        return logits

    def aiq_forward_static(self, scheme_bits, x, logits, stream=None):
        """aiq_forward on the library's built-in workspace.  `logits` must be provided by the
        caller ([batch][n_classes] float32 CUDA tensor): this call allocates nothing."""
        scheme = np.ascontiguousarray(scheme_bits, dtype=np.uint8)
        if scheme.shape != (self.n_layers,):
            raise ValueError("scheme length must equal the number of layers")
        _check(lib.aiq_forward_static(self.handle, _host(scheme), _dev(x), int(x.shape[0]),
                                      _dev(logits), _stream(stream)))
        return logits

    def aiq_eval_schemes(self, schemes, x, labels, preds=None, workspace=None, chunk=1024,
                         stream=None):
        schemes = np.ascontiguousarray(schemes, dtype=np.uint8)
        if schemes.ndim != 2 or schemes.shape[1] != self.n_layers:
            raise ValueError("schemes must be [S][L]")
        S, N = schemes.shape[0], x.shape[0]
        acc = np.zeros(S, dtype=np.float32)
        counts = np.zeros(S, dtype=np.int32)
        ws = workspace if workspace is not None else self.workspace(min(chunk, N), S)
        _check(lib.aiq_eval_schemes(self.handle, _host(schemes), S, _dev(x), _dev(labels), N,
                                    _host(acc), _host(counts), _dev(preds), _dev(ws), ws.numel(),
                                    _stream(stream)))
        return acc, counts

    def _search(self, which, x, labels, lam, options, layers, max_passes, workspace, chunk, stream):
        options = np.ascontiguousarray(options, dtype=np.uint8)
        n_sel = self.n_layers if layers is None else len(layers)
        lay = None if layers is None else np.ascontiguousarray(layers, dtype=np.int32)
        N = x.shape[0]
        ws = workspace if workspace is not None else self.workspace(min(chunk, N), max(1, n_sel * len(options)))
        scheme = np.zeros(self.n_layers, dtype=np.uint8)
        cap = 4 * (n_sel + 1) * max(1, max_passes)
        trace = (SearchStep * cap)()
        n_trace = C.c_int(0)
        if which == "greedy":
            _check(lib.aiq_search_greedy(self.handle, _host(lay), n_sel, _host(options), len(options), float(lam),
                                         _dev(x), _dev(labels), N, _host(scheme), trace, cap, C.byref(n_trace),
                                         _dev(ws), ws.numel(), _stream(stream)))
        else:
            _check(lib.aiq_search_coordinate_descent(self.handle, _host(lay), n_sel, _host(options), len(options),
                                                     float(lam), int(max_passes), _dev(x), _dev(labels), N,
                                                     _host(scheme), trace, cap, C.byref(n_trace), _dev(ws),
                                                     ws.numel(), _stream(stream)))
        steps = [dict(layer=t.layer, bits=t.bits, accepted=t.accepted, candidates=t.candidates, loss=t.loss,
                      acc=t.acc, ai=t.ai) for t in trace[:min(n_trace.value, cap)]]
        return scheme, steps

    def aiq_search_greedy(self, x, labels, lam, options=(8, 4), layers=None, workspace=None, chunk=1024,
                          stream=None):
        return self._search("greedy", x, labels, lam, options, layers, 1, workspace, chunk, stream)

    def aiq_search_coordinate_descent(self, x, labels, lam, options=(32, 8, 4), layers=None, max_passes=8,
                                      workspace=None, chunk=1024, stream=None):
        return self._search("cd", x, labels, lam, options, layers, max_passes, workspace, chunk, stream)

    def aiq_model_status(self, stream=None):
        _check(lib.aiq_model_status(self.handle, _stream(stream)))

    def aiq_debug_expire_wait(self, limit_cycles, stream=None):
        _check(lib.aiq_debug_expire_wait(self.handle, int(limit_cycles), _stream(stream)))

    def aiq_scheme_ai(self, scheme_bits, ai_batch=1):
        scheme = np.ascontiguousarray(scheme_bits, dtype=np.uint8)
        if scheme.shape != (self.n_layers,):
            raise ValueError("scheme length must equal the number of layers")
        ai, fl, by = C.c_double(), C.c_double(), C.c_double()
        _check(lib.aiq_scheme_ai(self.handle, _host(scheme), int(ai_batch), C.byref(ai), C.byref(fl),
                                 C.byref(by)))
        return ai.value, fl.value, by.value


def _f32():
    import torch
    return torch.float32
