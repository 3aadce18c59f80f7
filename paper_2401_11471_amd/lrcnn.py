"""ctypes binding of liblrcnn.so (include/lrcnn.h): argument marshalling only.

Every step of row-centric training runs in the HIP library; this module
converts Python values and torch tensors into the C ABI's plain pointers and
sizes. Device memory comes from torch; streams are torch's current stream.
If the library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os

# torch first: it brings its own HIP runtime, and liblrcnn.so must bind to
# that same runtime (one HIP/HSA runtime per process). Loading the library
# first would load the system runtime and leave torch and the library on
# different ones.
import torch  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))
# (LRCNN_LIB_PATH: another build of the library, e.g. a variant under test)
LIB_PATH = os.environ.get("LRCNN_LIB_PATH") or os.path.join(HERE, "liblrcnn.so")

OP_INPUT, OP_CONV, OP_MAXPOOL, OP_ADD = 0, 1, 2, 3
F32, BF16 = 0, 1
CARRY, RECOMPUTE = 0, 1
EVEN, BALANCED, EXPLICIT, PAPER_2PS = 0, 1, 2, 3
HYBRID_AUTO = -1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = -1, 0, 1, 2, 3

STATUS = {0: "OK", -1: "EINVAL", -2: "ESHAPE", -3: "EPARTITION",
          -4: "EWORKSPACE", -5: "ESTATE", -6: "EDTYPE", -7: "EHIP",
          -8: "EINFEASIBLE"}


class LrcnnError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class Node(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("op", "in0", "in1", "c_out", "kh", "kw",
                                         "sh", "sw", "ph", "pw", "affine", "relu")]


class Config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("in_c", C.c_int32), ("in_h", C.c_int32),
                ("in_w", C.c_int32), ("dtype", C.c_int32), ("mode", C.c_int32),
                ("n_bands", C.c_int32), ("policy", C.c_int32),
                ("bounds", C.POINTER(C.c_int32)), ("bp_refine", C.c_int32),
                ("hybrid_from", C.c_int32), ("first_rows", C.c_int32)]


class PlanInfo(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("n_bands", C.c_int32), ("mode", C.c_int32),
                ("dtype", C.c_int32), ("out_h", C.c_int32), ("out_w", C.c_int32),
                ("out_c", C.c_int32),
                ("workspace_bytes", C.c_size_t), ("layerwise_workspace_bytes", C.c_size_t),
                ("strip_bytes", C.c_size_t), ("band_cache_bytes", C.c_size_t),
                ("delta_bytes", C.c_size_t), ("carry_bytes", C.c_size_t),
                ("partial_bytes", C.c_size_t),
                ("omega_bytes", C.c_double), ("omega_fp_bytes", C.c_double),
                ("omega_bp_bytes", C.c_double), ("flops_tau", C.c_double),
                ("flops_rows", C.c_double), ("flops_layerwise", C.c_double),
                ("shared_rows", C.c_int64), ("halo_rows", C.c_int64),
                ("bp_bands", C.c_int32), ("fp_window_bytes", C.c_size_t),
                ("hybrid_from", C.c_int32)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


class Budget(C.Structure):
    _fields_ = [("budget_bytes", C.c_size_t), ("max_bands", C.c_int32),
                ("max_refine", C.c_int32), ("want_dx", C.c_int32)]


_BLOCK_EXPORTS = ("lrcnn_act8_bytes", "lrcnn_act8_pack", "lrcnn_act8_unpack",
                  "lrcnn_layer_norm_forward", "lrcnn_layer_norm_workspace_bytes",
                  "lrcnn_layer_norm_backward", "lrcnn_activation_forward",
                  "lrcnn_activation_backward", "lrcnn_linear_wgrad_workspace_bytes",
                  "lrcnn_linear_wgrad", "lrcnn_group_norm_workspace_bytes",
                  "lrcnn_group_norm_forward", "lrcnn_group_norm_backward", "lrcnn_dropout",
                  "lrcnn_gated_ffn_forward", "lrcnn_gated_ffn_backward")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build the HIP library first "
            "(python -c 'import __graft_entry__ as g; g.build()')")
    lib = C.CDLL(LIB_PATH)
    vp, sz, i32 = C.c_void_p, C.c_size_t, C.c_int32
    pp = C.POINTER(C.c_void_p)
    lib.lrcnn_plan.argtypes = [C.POINTER(Node), i32, C.POINTER(Config), C.POINTER(vp)]
    lib.lrcnn_plan_query.argtypes = [vp, C.POINTER(PlanInfo)]
    lib.lrcnn_plan_node_shape.argtypes = [vp, i32, C.POINTER(i32)]
    lib.lrcnn_plan_band_rows.argtypes = [vp, i32, i32, i32, C.POINTER(i32)]
    lib.lrcnn_plan_destroy.argtypes = [vp]
    lib.lrcnn_plan_step_bytes.argtypes = [vp, i32, i32, C.POINTER(sz)]
    lib.lrcnn_plan_for_budget.argtypes = [C.POINTER(Node), i32, C.POINTER(Config),
                                          C.POINTER(Budget), C.POINTER(vp)]
    lib.lrcnn_max_batch.argtypes = [C.POINTER(Node), i32, C.POINTER(Config), i32,
                                    C.POINTER(Budget), C.POINTER(i32)]
    lib.lrcnn_plan_destroy.restype = None
    lib.lrcnn_forward_rows.argtypes = [vp, vp, pp, pp, pp, vp, vp, sz, pp, vp]
    lib.lrcnn_forward_rows_static.argtypes = [vp, vp, pp, pp, pp, vp, pp, vp]
    lib.lrcnn_backward_rows.argtypes = [vp, vp, pp, pp, pp, vp, pp, vp, vp, sz, vp]
    lib.lrcnn_layerwise_reference_gpu.argtypes = [vp, vp, pp, pp, pp, vp, vp, pp, vp,
                                                  vp, sz, pp, vp]
    lib.lrcnn_head_workspace_bytes.argtypes = [vp, i32, C.POINTER(sz)]
    lib.lrcnn_head_loss.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lrcnn_sgd_update.argtypes = [vp, C.c_float, pp, pp, vp, vp, vp, vp, i32, vp]
    i64, f32, psz = C.c_int64, C.c_float, C.POINTER(sz)
    lib.lrcnn_act8_bytes.argtypes = [i64, i64, psz]
    lib.lrcnn_act8_pack.argtypes = [i64, i64, i32, vp, i64, vp, vp]
    lib.lrcnn_act8_unpack.argtypes = [i64, i64, i32, vp, vp, i64, vp]
    lib.lrcnn_layer_norm_forward.argtypes = [i64, i64, i32, vp, i64, vp, i64, vp, vp, f32, vp,
                                             i64, vp, i64, vp, vp, vp, vp]
    lib.lrcnn_layer_norm_workspace_bytes.argtypes = [i64, i64, psz]
    lib.lrcnn_layer_norm_backward.argtypes = [i64, i64, i32, vp, i64, vp, i64, vp, vp, vp, vp,
                                              vp, i64, vp, i64, vp, vp, i32, vp, sz, vp]
    lib.lrcnn_activation_forward.argtypes = [i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp,
                                             vp, vp, vp]
    lib.lrcnn_activation_backward.argtypes = [i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp,
                                              vp, vp, i64, vp, i64, vp, vp]
    lib.lrcnn_linear_wgrad_workspace_bytes.argtypes = [i64, i64, i64, i32, psz]
    lib.lrcnn_linear_wgrad.argtypes = [i64, i64, i64, i32, vp, i64, vp, vp, vp, vp, vp, i32, vp,
                                       sz, vp]
    lib.lrcnn_group_norm_workspace_bytes.argtypes = [i64, i64, i64, i64, psz]
    lib.lrcnn_group_norm_forward.argtypes = [i64, i64, i64, i64, i32, i32, vp, i64, vp, vp, f32,
                                             vp, i64, vp, vp, vp, vp, sz, vp]
    lib.lrcnn_group_norm_backward.argtypes = [i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp,
                                              vp, vp, vp, vp, vp, i64, vp, vp, i32, vp, sz, vp]
    lib.lrcnn_dropout.argtypes = [i64, i64, i32, vp, i64, vp, i64, C.c_double, vp, i32, i64, vp,
                                  i64, vp]
    lib.lrcnn_gated_ffn_forward.argtypes = [i64, i64, i64, i64, i32, i32, vp, i64, vp, vp, vp, i64,
                                            vp, i64, vp, vp, vp, vp, vp, i64, vp]
    lib.lrcnn_gated_ffn_backward.argtypes = [i64, i64, i64, i64, i32, i32, vp, i64, vp, vp, i64,
                                             vp, vp, vp, i64, vp, vp, vp, i64, vp]
    lib.lrcnn_last_error.restype = C.c_char_p
    lib.lrcnn_debug_dry_run.argtypes = [C.c_int]
    lib.lrcnn_debug_dry_run.restype = None
    lib.lrcnn_debug_fp_pipeline.argtypes = [C.c_int]
    lib.lrcnn_debug_fp_pipeline.restype = None
    lib.lrcnn_debug_act_fusion.argtypes = [C.c_int]
    lib.lrcnn_debug_act_fusion.restype = None
    lib.lrcnn_debug_serial_wgrad.argtypes = [C.c_int]
    lib.lrcnn_debug_serial_wgrad.restype = None
    lib.lrcnn_debug_fork_wgrad.argtypes = [C.c_int]
    lib.lrcnn_debug_fork_wgrad.restype = C.c_int
    lib.lrcnn_debug_dgrad_phases.argtypes = [C.c_int]
    lib.lrcnn_debug_dgrad_phases.restype = None
    lib.lrcnn_debug_ffn_tile.argtypes = [i32]
    lib.lrcnn_debug_ffn_tile.restype = None
    lib.lrcnn_debug_profile.argtypes = [C.c_int]
    lib.lrcnn_debug_profile.restype = None
    lib.lrcnn_debug_profile_collect.restype = C.c_int
    lib.lrcnn_debug_profile_entry.argtypes = [i32, C.POINTER(C.c_char_p),
                                              C.POINTER(C.c_int64),
                                              C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.lrcnn_debug_profile_entry.restype = C.c_int
    lib.lrcnn_debug_profile_roofline.argtypes = [i32, C.POINTER(C.c_double),
                                                 C.POINTER(C.c_double)]
    lib.lrcnn_debug_profile_roofline.restype = C.c_int
    lib.lrcnn_debug_layerwise_map.argtypes = [vp, i32, C.POINTER(sz)]
    lib.lrcnn_debug_layerwise_map.restype = C.c_int
    for f in ("lrcnn_plan", "lrcnn_plan_query", "lrcnn_plan_node_shape",
              "lrcnn_plan_band_rows", "lrcnn_forward_rows", "lrcnn_forward_rows_static",
              "lrcnn_backward_rows",
              "lrcnn_layerwise_reference_gpu", "lrcnn_plan_step_bytes",
              "lrcnn_plan_for_budget", "lrcnn_max_batch", "lrcnn_head_workspace_bytes",
              "lrcnn_head_loss", "lrcnn_sgd_update", *_BLOCK_EXPORTS):
        getattr(lib, f).restype = C.c_int
    return lib


LIB = _load()

# Names the header declares (checked by the tests against the shared object).
EXPORTS = ("lrcnn_plan", "lrcnn_plan_query", "lrcnn_plan_node_shape",
           "lrcnn_plan_band_rows", "lrcnn_plan_destroy", "lrcnn_plan_step_bytes",
           "lrcnn_plan_for_budget", "lrcnn_max_batch", "lrcnn_head_workspace_bytes",
           "lrcnn_head_loss", "lrcnn_sgd_update", "lrcnn_forward_rows",
           "lrcnn_forward_rows_static",
           "lrcnn_backward_rows", "lrcnn_layerwise_reference_gpu", "lrcnn_last_error",
           "lrcnn_debug_dry_run", "lrcnn_debug_fp_pipeline", "lrcnn_debug_act_fusion",
           "lrcnn_debug_dgrad_phases", "lrcnn_debug_serial_wgrad",
           "lrcnn_debug_fork_wgrad", "lrcnn_debug_ffn_tile",
           "lrcnn_debug_profile",
           "lrcnn_debug_profile_collect", "lrcnn_debug_profile_entry",
           "lrcnn_debug_profile_roofline",
           "lrcnn_debug_layerwise_map", *_BLOCK_EXPORTS)


def _check(code):
    if code != 0:
        raise LrcnnError(code, LIB.lrcnn_last_error().decode())


class Plan:
    """Owns an lrcnn_plan_t handle."""

    def __init__(self, handle, nodes):
        self.handle = handle
        self.nodes = list(nodes)
        self.n = len(self.nodes)

    def __del__(self):
        if getattr(self, "handle", None) and LIB is not None:
            LIB.lrcnn_plan_destroy(self.handle)
            self.handle = None

    def info(self):
        inf = PlanInfo()
        _check(LIB.lrcnn_plan_query(self.handle, C.byref(inf)))
        return inf.as_dict()

    def node_shape(self, v):
        out = (C.c_int32 * 3)()
        _check(LIB.lrcnn_plan_node_shape(self.handle, v, out))
        return tuple(out)

    def step_bytes(self, layerwise=False, want_dx=False):
        """Workspace plus every other buffer of one step (the xi of
        Eqs. (9)-(10)), in bytes."""
        out = C.c_size_t()
        _check(LIB.lrcnn_plan_step_bytes(self.handle, 1 if layerwise else 0,
                                         1 if want_dx else 0, C.byref(out)))
        return out.value

    def band_rows(self, band, v, phase=1):
        """Rows (a, b, lo, hi) of node v in a backward (phase 1) or forward
        (phase 0) band."""
        out = (C.c_int32 * 4)()
        _check(LIB.lrcnn_plan_band_rows(self.handle, phase, band, v, out))
        return tuple(out)


def lrcnn_plan(nodes, batch, in_c, in_h, in_w, dtype=F32, mode=CARRY, n_bands=1,
               policy=EVEN, bounds=None, bp_refine=1, hybrid_from=0, first_rows=0):
    arr = (Node * len(nodes))(*[Node(*nd) for nd in nodes])
    cfg = Config(batch, in_c, in_h, in_w, dtype, mode, n_bands, policy, None, bp_refine,
                 hybrid_from, first_rows)
    keep = None
    if bounds is not None:
        keep = (C.c_int32 * len(bounds))(*bounds)
        cfg.bounds = C.cast(keep, C.POINTER(C.c_int32))
    h = C.c_void_p()
    _check(LIB.lrcnn_plan(arr, len(nodes), C.byref(cfg), C.byref(h)))
    return Plan(h, nodes)


def _node_cfg(nodes, batch, in_c, in_h, in_w, dtype, mode, n_bands, policy, bp_refine,
              hybrid_from, first_rows=0):
    arr = (Node * len(nodes))(*[Node(*nd) for nd in nodes])
    return arr, Config(batch, in_c, in_h, in_w, dtype, mode, n_bands, policy, None,
                       bp_refine, hybrid_from, first_rows)


def lrcnn_plan_for_budget(nodes, batch, in_c, in_h, in_w, budget_bytes, dtype=F32,
                          mode=CARRY, policy=EVEN, max_bands=0, max_refine=1,
                          want_dx=False, hybrid_from=0):
    """Smallest (N_BP, N_FP) whose step fits budget_bytes (Eqs. (9)-(10))."""
    arr, cfg = _node_cfg(nodes, batch, in_c, in_h, in_w, dtype, mode, 1, policy, 1,
                         hybrid_from)
    bud = Budget(int(budget_bytes), max_bands, max_refine, 1 if want_dx else 0)
    h = C.c_void_p()
    _check(LIB.lrcnn_plan_for_budget(arr, len(nodes), C.byref(cfg), C.byref(bud),
                                     C.byref(h)))
    return Plan(h, nodes)


def lrcnn_max_batch(nodes, in_c, in_h, in_w, budget_bytes, dtype=F32, mode=CARRY,
                    n_bands=1, policy=EVEN, bp_refine=1, hybrid_from=0, layerwise=False,
                    want_dx=False):
    """Largest batch whose row-centric (or layer-wise) step fits budget_bytes."""
    arr, cfg = _node_cfg(nodes, 1, in_c, in_h, in_w, dtype, mode, n_bands, policy,
                         bp_refine, hybrid_from)
    bud = Budget(int(budget_bytes), 0, 1, 1 if want_dx else 0)
    out = C.c_int32()
    _check(LIB.lrcnn_max_batch(arr, len(nodes), C.byref(cfg), 1 if layerwise else 0,
                               C.byref(bud), C.byref(out)))
    return out.value


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _ptr_array(ts):
    return (C.c_void_p * len(ts))(*[None if t is None else t.data_ptr() for t in ts])


def _stream(stream):
    if stream is not None:
        return C.c_void_p(stream)
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream(stream, like):
    """The stream as a number: torch's current one of the tensors' device, asked
    for without making a Stream object (1 us of a call's 8). The last thing a
    call asks for: neither host memory goes further nor another GPU's. (Launches
    go to the current device, and the default stream is 0 on each.)"""
    dev = like[2]
    if dev < 0:
        _einval("the tensors must be on a GPU")
    if dev != torch._C._cuda_getDevice():
        _einval(f"the tensors are on cuda:{dev}, which is not the current device")
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream


def lrcnn_forward_rows(plan, x, weights, scales, shifts, y, workspace, masks=None,
                       stream=None):
    """weights/scales/shifts/masks: per-node lists (None where unused)."""
    _check(LIB.lrcnn_forward_rows(
        plan.handle, _ptr(x), _ptr_array(weights), _ptr_array(scales),
        _ptr_array(shifts), _ptr(y), _ptr(workspace), workspace.numel(),
        _ptr_array(masks) if masks is not None else None, _stream(stream)))


def lrcnn_forward_rows_static(plan, x, weights, scales, shifts, y, masks=None, stream=None):
    """lrcnn_forward_rows on the library's static device workspace (no
    workspace argument; the call allocates nothing)."""
    _check(LIB.lrcnn_forward_rows_static(
        plan.handle, _ptr(x), _ptr_array(weights), _ptr_array(scales),
        _ptr_array(shifts), _ptr(y),
        _ptr_array(masks) if masks is not None else None, _stream(stream)))


STATIC_WORKSPACE_BYTES = 64 << 20


def lrcnn_backward_rows(plan, x, weights, scales, shifts, dy, dws, dx, workspace,
                        stream=None):
    _check(LIB.lrcnn_backward_rows(
        plan.handle, _ptr(x), _ptr_array(weights), _ptr_array(scales),
        _ptr_array(shifts), _ptr(dy), _ptr_array(dws), _ptr(dx), _ptr(workspace),
        workspace.numel(), _stream(stream)))


def lrcnn_layerwise_reference_gpu(plan, x, weights, scales, shifts, dy, y, dws, dx,
                                  workspace, masks=None, stream=None):
    _check(LIB.lrcnn_layerwise_reference_gpu(
        plan.handle, _ptr(x), _ptr_array(weights), _ptr_array(scales),
        _ptr_array(shifts), _ptr(dy), _ptr(y), _ptr_array(dws), _ptr(dx),
        _ptr(workspace), workspace.numel(),
        _ptr_array(masks) if masks is not None else None, _stream(stream)))


def lrcnn_head_workspace_bytes(plan, n_classes):
    out = C.c_size_t()
    _check(LIB.lrcnn_head_workspace_bytes(plan.handle, n_classes, C.byref(out)))
    return out.value


def lrcnn_head_loss(plan, y, fc_w, fc_b, labels, logits, loss, dy, d_fc_w, d_fc_b, head_ws,
                    stream=None):
    """Classifier head + softmax cross-entropy: logits, loss, dL/dy, head
    gradients (all device tensors; n_classes = fc_w.shape[0])."""
    _check(LIB.lrcnn_head_loss(
        plan.handle, _ptr(y), _ptr(fc_w), _ptr(fc_b), _ptr(labels), fc_w.shape[0],
        _ptr(logits), _ptr(loss), _ptr(dy), _ptr(d_fc_w), _ptr(d_fc_b), _ptr(head_ws),
        head_ws.numel(), _stream(stream)))


def lrcnn_sgd_update(plan, lr, weights, dws, fc_w=None, d_fc_w=None, fc_b=None, d_fc_b=None,
                     stream=None):
    """theta -= lr * g for every conv weight and (when given) the head."""
    n_classes = fc_w.shape[0] if fc_w is not None else 0
    _check(LIB.lrcnn_sgd_update(
        plan.handle, C.c_float(lr), _ptr_array(weights), _ptr_array(dws), _ptr(fc_w),
        _ptr(d_fc_w), _ptr(fc_b), _ptr(d_fc_b), n_classes, _stream(stream)))


# ---- feed-forward blocks with 8-bit activation checkpoints (2-d tensors of one
# dtype and device, columns next to each other, rows at any stride). The tensors'
# shapes give the sizes; ones that do not agree, or are not on the current GPU, are
# refused before the call.
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _einval(msg):
    raise LrcnnError(-1, msg)


def _first(name, t):
    """(shape, dtype, device index, library dtype, pointer, row stride) of the
    matrix that the call's other tensors have to agree with."""
    shape, dtype = t.shape, t.dtype
    if len(shape) != 2:
        _einval(f"{name} must have two dimensions")
    if shape[1] < 1:
        raise LrcnnError(-2, f"{name} has no columns")
    code = _DTYPES.get(dtype)
    if code is None:
        raise LrcnnError(-6, f"{name}: dtype must be float32 or bfloat16")
    like = (shape, dtype, t.get_device())
    return (*like, code, t.data_ptr(), _ld(name, t))


def _ld(name, t):
    """Row stride of a matrix (0: dense)."""
    if t.is_contiguous():
        return 0
    rows, cols = t.shape
    ld, one = t.stride()
    if (one != 1 and cols > 1) or (ld < cols and rows > 1):
        _einval(f"{name}: columns must be next to each other, rows apart")
    return ld if rows > 1 else 0


def _mat(name, t, like):
    """Pointer and row stride of a matrix of the first one's shape, dtype and device
    (None: absent)."""
    if t is None:
        return None, 0
    if t.shape != like[0] or t.dtype is not like[1] or t.get_device() != like[2]:
        _einval(f"{name} must be a matrix {tuple(like[0])} of {like[1]} on the same device")
    return t.data_ptr(), _ld(name, t)


def _vec(name, t, n, like):
    """Pointer of a dense float32 vector of n elements (None: absent)."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous() \
            or t.get_device() != like[2]:
        _einval(f"{name} must be {n} dense float32 values on the same device")
    return t.data_ptr()


def _bytes(name, t, like):
    """Pointer and size of a byte buffer (None: absent)."""
    if t is None:
        return None, 0
    if t.dtype is not torch.uint8 or not t.is_contiguous() or t.get_device() != like[2]:
        _einval(f"{name} must be dense uint8 on the same device")
    return t.data_ptr(), t.numel()


def _workspace(t, like, need, *sizes):
    """Pointer and size of a workspace. The library refuses one that is too small;
    of tensors that do not get that far it is said here."""
    p, n = _bytes("workspace", t, like)
    if t is not None and like[2] < 0 and n < need(*sizes):
        raise LrcnnError(-4, f"workspace needs {need(*sizes)} bytes, got {n}")
    return p, n


def _ckpt(name, t, shape, like):
    """Pointer of the checkpoint of a matrix of that shape (None: absent)."""
    if t is None:
        return None
    p, n = _bytes(name, t, like)
    codes = shape[0] * (shape[1] + 31 & -32)
    if n < (codes + 255 & -256) + (codes // 32 + 255 & -256):
        _einval(f"{name} is smaller than the checkpoint of {tuple(shape)}")
    return p


def _query(fn, *args):
    out = C.c_size_t()
    _check(fn(*args, C.byref(out)))
    return out.value


def lrcnn_act8_bytes(rows, cols):
    """Bytes of the 8-bit checkpoint of a rows x cols matrix."""
    return _query(LIB.lrcnn_act8_bytes, rows, cols)


def lrcnn_act8_pack(x, ckpt, stream=None):
    """ckpt (uint8, lrcnn_act8_bytes) = the 8-bit checkpoint of x."""
    like = _first("x", x)
    shape, _, _, dt, px, ldx = like
    _check(LIB.lrcnn_act8_pack(shape[0], shape[1], dt, px, ldx, _ckpt("ckpt", ckpt, shape, like),
                               _raw_stream(stream, like)))


def lrcnn_act8_unpack(ckpt, y, stream=None):
    """y = what the checkpoint of a matrix of y's shape stands for."""
    like = _first("y", y)
    shape, _, _, dt, py, ldy = like
    _check(LIB.lrcnn_act8_unpack(shape[0], shape[1], dt, _ckpt("ckpt", ckpt, shape, like), py, ldy,
                                 _raw_stream(stream, like)))


def lrcnn_layer_norm_forward(x, gamma, beta, eps, y, residual=None, total=None, mean=None,
                             rstd=None, ckpt=None, stream=None):
    """y = layer norm of the rows of x (+ residual: their sum goes to total);
    mean, rstd per row; ckpt: the checkpoint of the normalised rows."""
    like = _first("x", x)
    shape, _, _, dt, px, ldx = like
    rows, cols = shape
    pr, ldr = _mat("residual", residual, like)
    pt, ldt = _mat("total", total, like)
    py, ldy = _mat("y", y, like)
    _check(LIB.lrcnn_layer_norm_forward(
        rows, cols, dt, px, ldx, pr, ldr, _vec("gamma", gamma, cols, like),
        _vec("beta", beta, cols, like), eps, pt, ldt, py, ldy, _vec("mean", mean, rows, like),
        _vec("rstd", rstd, rows, like), _ckpt("ckpt", ckpt, shape, like), _raw_stream(stream, like)))


def lrcnn_layer_norm_workspace_bytes(rows, cols):
    return _query(LIB.lrcnn_layer_norm_workspace_bytes, rows, cols)


def lrcnn_layer_norm_backward(dy, rstd, gamma, dx, dgamma=None, dbeta=None, workspace=None,
                              x=None, mean=None, ckpt=None, dres=None, accumulate=False,
                              stream=None):
    """dx (+ dres), dgamma and dbeta from dy and either (x, mean) or ckpt."""
    like = _first("dy", dy)
    shape, _, _, dt, pdy, lddy = like
    rows, cols = shape
    px, ldx = _mat("x", x, like)
    pr, ldr = _mat("dres", dres, like)
    pdx, lddx = _mat("dx", dx, like)
    pw, nw = _workspace(workspace, like, lrcnn_layer_norm_workspace_bytes, rows, cols)
    _check(LIB.lrcnn_layer_norm_backward(
        rows, cols, dt, pdy, lddy, px, ldx, _vec("mean", mean, rows, like),
        _ckpt("ckpt", ckpt, shape, like), _vec("rstd", rstd, rows, like),
        _vec("gamma", gamma, cols, like), pr, ldr, pdx, lddx, _vec("dgamma", dgamma, cols, like),
        _vec("dbeta", dbeta, cols, like), 1 if accumulate else 0, pw, nw, _raw_stream(stream, like)))


def lrcnn_activation_forward(kind, u, a=None, v=None, ckpt_u=None, ckpt_v=None, ckpt_a=None,
                             stream=None):
    """a = f(u) (times v), and the checkpoints of u, v and a that are given."""
    like = _first("u", u)
    shape, _, _, dt, pu, ldu = like
    pv, ldv = _mat("v", v, like)
    pa, lda = _mat("a", a, like)
    _check(LIB.lrcnn_activation_forward(
        shape[0], shape[1], dt, kind, pu, ldu, pv, ldv, pa, lda,
        _ckpt("ckpt_u", ckpt_u, shape, like), _ckpt("ckpt_v", ckpt_v, shape, like),
        _ckpt("ckpt_a", ckpt_a, shape, like), _raw_stream(stream, like)))


def lrcnn_activation_backward(kind, da, du, u=None, v=None, ckpt_u=None, ckpt_v=None, dv=None,
                              ckpt_a=None, stream=None):
    """du (and dv) from da and either u (and v) or their checkpoints; ckpt_a:
    receives the checkpoint of the activation's output."""
    like = _first("da", da)
    shape, _, _, dt, pda, ldda = like
    pu, ldu = _mat("u", u, like)
    pv, ldv = _mat("v", v, like)
    pdu, lddu = _mat("du", du, like)
    pdv, lddv = _mat("dv", dv, like)
    _check(LIB.lrcnn_activation_backward(
        shape[0], shape[1], dt, kind, pda, ldda, pu, ldu, pv, ldv,
        _ckpt("ckpt_u", ckpt_u, shape, like), _ckpt("ckpt_v", ckpt_v, shape, like), pdu, lddu,
        pdv, lddv, _ckpt("ckpt_a", ckpt_a, shape, like), _raw_stream(stream, like)))


def lrcnn_linear_wgrad_workspace_bytes(rows, n_in, n_out, dtype=F32):
    return _query(LIB.lrcnn_linear_wgrad_workspace_bytes, rows, n_in, n_out, dtype)


def lrcnn_linear_wgrad(dy, ckpt, dw, workspace=None, db=None, scale=None, shift=None,
                       accumulate=False, stream=None):
    """dw [n_out][n_in] and db [n_out] of a linear layer from dy [rows][n_out] and
    the checkpoint [rows][n_in] of its input (the input being scale times that
    plus shift, per column)."""
    like = _first("dy", dy)
    (rows, n_out), _, _, dt, pdy, lddy = like
    if dw.dim() != 2 or dw.shape[0] != n_out:
        _einval("dw must be [n_out][n_in]")
    n_in = dw.shape[1]
    pw, nw = _workspace(workspace, like, lrcnn_linear_wgrad_workspace_bytes, rows, n_in, n_out,
                        dt)
    _check(LIB.lrcnn_linear_wgrad(
        rows, n_in, n_out, dt, pdy, lddy, _ckpt("ckpt", ckpt, (rows, n_in), like),
        _vec("scale", scale, n_in, like), _vec("shift", shift, n_in, like),
        _vec("dw", dw, n_out * n_in, like), _vec("db", db, n_out, like), 1 if accumulate else 0,
        pw, nw, _raw_stream(stream, like)))


# ---- group norm of a feature map, dropout, the gated feed-forward block
def _rows(name, t, cols, like):
    """Pointer and row stride of a matrix of the first one's rows, dtype and device and
    `cols` columns (None: absent)."""
    if t is None:
        return None, 0
    if t.shape != (like[0][0], cols) or t.dtype is not like[1] or t.get_device() != like[2]:
        _einval(f"{name} must be a matrix {(like[0][0], cols)} of {like[1]} on the same device")
    return t.data_ptr(), _ld(name, t)


def _weight(name, t, n_out, n_in, like):
    """Pointer of a dense weight [n_out][n_in] of the matrices' dtype (None: absent)."""
    if t is None:
        return None
    if t.shape != (n_out, n_in) or t.dtype is not like[1] or t.get_device() != like[2] \
            or not t.is_contiguous():
        _einval(f"{name} must be dense [{n_out}][{n_in}] of {like[1]} on the same device")
    return t.data_ptr()


def _images(shape, batch):
    """Pixels of each of the `batch` images whose rows a matrix holds."""
    if batch < 0 or (shape[0] % batch if batch else shape[0]):
        _einval(f"{shape[0]} rows are not {batch} images of as many pixels")
    return shape[0] // batch if batch else 0


def lrcnn_group_norm_workspace_bytes(batch, pixels, channels, groups):
    return _query(LIB.lrcnn_group_norm_workspace_bytes, batch, pixels, channels, groups)


def lrcnn_group_norm_forward(kind, x, gamma, beta, eps, y, batch, groups, workspace, mean=None,
                             rstd=None, ckpt=None, stream=None):
    """y = f(group norm of x), f of `kind` (ACT_NONE: x itself); x: [batch * pixels]
    [channels]; mean, rstd per image and group; ckpt: the checkpoint of the
    normalised map."""
    like = _first("x", x)
    shape, _, _, dt, px, ldx = like
    cols, pixels = shape[1], _images(shape, batch)
    py, ldy = _mat("y", y, like)
    pw, nw = _workspace(workspace, like, lrcnn_group_norm_workspace_bytes, batch, pixels, cols,
                        groups)
    _check(LIB.lrcnn_group_norm_forward(
        batch, pixels, cols, groups, dt, kind, px, ldx, _vec("gamma", gamma, cols, like),
        _vec("beta", beta, cols, like), eps, py, ldy, _vec("mean", mean, batch * groups, like),
        _vec("rstd", rstd, batch * groups, like), _ckpt("ckpt", ckpt, shape, like), pw, nw,
        _raw_stream(stream, like)))


def lrcnn_group_norm_backward(kind, dy, rstd, gamma, beta, dx, batch, groups, workspace,
                              dgamma=None, dbeta=None, x=None, mean=None, ckpt=None,
                              accumulate=False, stream=None):
    """dx, dgamma and dbeta from dy and either (x, mean) or ckpt."""
    like = _first("dy", dy)
    shape, _, _, dt, pdy, lddy = like
    cols, pixels = shape[1], _images(shape, batch)
    px, ldx = _mat("x", x, like)
    pdx, lddx = _mat("dx", dx, like)
    pw, nw = _workspace(workspace, like, lrcnn_group_norm_workspace_bytes, batch, pixels, cols,
                        groups)
    _check(LIB.lrcnn_group_norm_backward(
        batch, pixels, cols, groups, dt, kind, pdy, lddy, px, ldx,
        _vec("mean", mean, batch * groups, like), _ckpt("ckpt", ckpt, shape, like),
        _vec("rstd", rstd, batch * groups, like), _vec("gamma", gamma, cols, like),
        _vec("beta", beta, cols, like), pdx, lddx, _vec("dgamma", dgamma, cols, like),
        _vec("dbeta", dbeta, cols, like), 1 if accumulate else 0, pw, nw,
        _raw_stream(stream, like)))


def lrcnn_dropout(x, y, p, rng, residual=None, site=0, first_row=0, stream=None):
    """y = x with a share p of its elements dropped, the others over 1 - p
    (+ residual). rng: int64 [2] on the GPU, the seed and the offset; the same call
    on the gradient, without residual, is the backward pass."""
    like = _first("x", x)
    shape, _, _, dt, px, ldx = like
    pr, ldr = _mat("residual", residual, like)
    py, ldy = _mat("y", y, like)
    if rng.dtype is not torch.int64 or rng.numel() != 2 or not rng.is_contiguous() \
            or rng.get_device() != like[2]:
        _einval("rng must be two dense int64 values on the same device")
    _check(LIB.lrcnn_dropout(shape[0], shape[1], dt, px, ldx, pr, ldr, p, rng.data_ptr(), site,
                             first_row, py, ldy, _raw_stream(stream, like)))


def lrcnn_gated_ffn_forward(kind, x, w1, a, b1=None, w2=None, b2=None, z=None, uv=None,
                            ckpt_u=None, ckpt_v=None, stream=None):
    """a = f(x Wu^T + bu) * (x Wv^T + bv), w1 = [Wu; Wv], and with z: z = a w2^T + b2.
    uv, ckpt_u, ckpt_v: receive what the backward pass reads, full-width or as
    checkpoints."""
    like = _first("x", x)
    (rows, n_in), _, _, dt, px, ldx = like
    hidden = a.shape[-1]
    n_out = 0 if z is None else z.shape[-1]
    pa, lda = _rows("a", a, hidden, like)
    puv, lduv = _rows("uv", uv, 2 * hidden, like)
    pz, ldz = _rows("z", z, n_out, like)
    if (z is None) != (w2 is None) or (b2 is not None and z is None):
        _einval("z goes with w2 (and b2)")
    _check(LIB.lrcnn_gated_ffn_forward(
        rows, n_in, hidden, n_out, dt, kind, px, ldx, _weight("w1", w1, 2 * hidden, n_in, like),
        _vec("b1", b1, 2 * hidden, like), pa, lda, puv, lduv,
        _ckpt("ckpt_u", ckpt_u, (rows, hidden), like),
        _ckpt("ckpt_v", ckpt_v, (rows, hidden), like), _weight("w2", w2, n_out, hidden, like),
        _vec("b2", b2, n_out, like), pz, ldz, _raw_stream(stream, like)))


def lrcnn_gated_ffn_backward(kind, dz, w2t, duv, uv=None, ckpt_u=None, ckpt_v=None, ckpt_a=None,
                             w1t=None, dx=None, stream=None):
    """duv = [du dv] from dz, the transposed w2 and either uv or (ckpt_u, ckpt_v);
    ckpt_a: receives the checkpoint of f(u) * v; with dx: dx = duv W1, w1t the
    transposed w1."""
    like = _first("dz", dz)
    (rows, n_out), _, _, dt, pdz, lddz = like
    if w2t.dim() != 2:
        _einval("w2t must be [hidden][n_out]")
    hidden = w2t.shape[0]
    n_in = 0 if dx is None else dx.shape[-1]
    puv, lduv = _rows("uv", uv, 2 * hidden, like)
    pduv, ldduv = _rows("duv", duv, 2 * hidden, like)
    pdx, lddx = _rows("dx", dx, n_in, like)
    if (dx is None) != (w1t is None):
        _einval("dx goes with w1t")
    _check(LIB.lrcnn_gated_ffn_backward(
        rows, n_in, hidden, n_out, dt, kind, pdz, lddz, _weight("w2t", w2t, hidden, n_out, like),
        puv, lduv, _ckpt("ckpt_u", ckpt_u, (rows, hidden), like),
        _ckpt("ckpt_v", ckpt_v, (rows, hidden), like), pduv, ldduv,
        _ckpt("ckpt_a", ckpt_a, (rows, hidden), like),
        _weight("w1t", w1t, n_in, 2 * hidden, like), pdx, lddx, _raw_stream(stream, like)))


def lrcnn_debug_dry_run(on):
    """Test hook: walk schedules with all host checks but launch nothing."""
    LIB.lrcnn_debug_dry_run(1 if on else 0)


def lrcnn_debug_fp_pipeline(on):
    """Test hook: forward bands pipelined on two streams (on) or sequential (off,
    the default)."""
    LIB.lrcnn_debug_fp_pipeline(1 if on else 0)


def lrcnn_debug_serial_wgrad(on):
    """Test hook: all weight gradients on the caller's stream (on) or some on the
    plan's side stream beside the input gradients (off, the default)."""
    LIB.lrcnn_debug_serial_wgrad(1 if on else 0)


def lrcnn_debug_fork_wgrad(mode):
    """Test hook: weight gradients on the side stream (0 by estimate, other ones
    in a captured graph; 1 all, 2 every other one). Returns how many went there
    since the last call."""
    return LIB.lrcnn_debug_fork_wgrad(int(mode))


def lrcnn_debug_ffn_tile(tile):
    """Test hook: the gated feed-forward block's tile (-1 by estimate; 0 .. 7 as the
    header lists them, where the operands allow it)."""
    LIB.lrcnn_debug_ffn_tile(tile)


def lrcnn_debug_act_fusion(on):
    """Test hook: error operands formed by the consumer's input gradient (on) or
    by their own activation-backward pass (off)."""
    LIB.lrcnn_debug_act_fusion(1 if on else 0)


def lrcnn_debug_dgrad_phases(mode):
    """Test hook: strided input gradients by phase (0 estimate, 1 always, 2 never,
    3 always in separate launches, 4 always in one launch where there is one)."""
    LIB.lrcnn_debug_dgrad_phases(int(mode))


def lrcnn_debug_profile(on):
    """Test hook: time every matrix-core kernel launch with HIP events."""
    LIB.lrcnn_debug_profile(1 if on else 0)


def lrcnn_debug_profile_collect(roofline=False):
    """Per-kernel aggregate of the recorded launches (streams synchronised
    by the caller): {name: (launches, ms, flops)}, with roofline also the
    summed algorithmic bytes and roofline ms: (launches, ms, flops, bytes,
    roofline_ms)."""
    n = LIB.lrcnn_debug_profile_collect()
    if n < 0:
        raise LrcnnError(-7, "profile collection failed")
    out = {}
    for i in range(n):
        nm, la, ms, fl = C.c_char_p(), C.c_int64(), C.c_double(), C.c_double()
        LIB.lrcnn_debug_profile_entry(i, C.byref(nm), C.byref(la), C.byref(ms), C.byref(fl))
        if roofline:
            by, rf = C.c_double(), C.c_double()
            LIB.lrcnn_debug_profile_roofline(i, C.byref(by), C.byref(rf))
            out[nm.value.decode()] = (la.value, ms.value, fl.value, by.value, rf.value)
        else:
            out[nm.value.decode()] = (la.value, ms.value, fl.value)
    return out


def lrcnn_debug_layerwise_map(plan, node):
    """Test hook: byte offset of node's full map in the layer-wise workspace,
    or None where the map is not stored there (input, output, fused conv)."""
    out = C.c_size_t()
    code = LIB.lrcnn_debug_layerwise_map(plan.handle, node, C.byref(out))
    return out.value if code == 0 else None
