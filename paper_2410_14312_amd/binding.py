"""ctypes binding of libtmps.so: same names as the C ABI, argument marshalling only."""
import ctypes as C
import operator
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtmps.so")
_lib = None

TMPS_F32, TMPS_BF16_F32MASTER = 0, 1
TMPS_LINEAR, TMPS_CONV2D, TMPS_MAXPOOL, TMPS_SOFTMAX_CE, TMPS_LAYERNORM, TMPS_ATTENTION, TMPS_EMBEDDING = 1, 2, 3, 4, 5, 6, 7
TMPS_AFFINE, TMPS_RESADD, TMPS_AVGPOOL = 8, 9, 10
TMPS_ROTARY, TMPS_NORMJOIN, TMPS_DISTILL = 11, 12, 13
TMPS_FLAG_RELU, TMPS_FLAG_GELU, TMPS_FLAG_RMS, TMPS_FLAG_GATE, TMPS_FLAG_INTERLEAVED, TMPS_FLAG_OWN_LADDERS, TMPS_FLAG_SILU = 1, 2, 4, 8, 16, 32, 64


class TmpsError(RuntimeError):
    def __init__(self, code, text):
        super().__init__("libtmps error %d: %s" % (code, text))
        self.code = code


class LayerDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("dims", C.c_int32 * 8), ("flags", C.c_int32)]


class StageCfg(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("micro_batch", C.c_int32), ("n_micro", C.c_int32),
                ("max_stash", C.c_int32), ("is_last", C.c_int32), ("borrow_input", C.c_int32),
                ("lr", C.c_float), ("momentum", C.c_float)]


Axes = C.c_int32 * 3


class RotaryDesc(C.Structure):
    _fields_ = [("heads", C.c_int32), ("dh", C.c_int32), ("pairs", Axes), ("flags", C.c_int32), ("base", C.c_float)]


class DistillDesc(C.Structure):
    _fields_ = [("classes", C.c_int32), ("k", C.c_int32), ("temperature", C.c_float), ("alpha", C.c_float), ("grad_scale", C.c_float)]


class ScanDesc(C.Structure):
    _fields_ = [("heads", C.c_int32), ("dh", C.c_int32), ("groups", C.c_int32), ("n", C.c_int32)]


class Array(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32)]


_ARRAY = np.dtype({"names": ["data", "out", "n", "dtype"], "formats": ["u8", "u8", "i8", "i4"], "itemsize": C.sizeof(Array)})   # the same for numpy


EXPORTS = {
    "tmps_stage_bytes": (C.c_int, [C.POINTER(LayerDesc), C.c_int, C.POINTER(StageCfg), C.POINTER(C.c_size_t),
                                   C.POINTER(C.c_size_t), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "tmps_stage_create": (C.c_int, [C.POINTER(C.c_void_p), C.POINTER(LayerDesc), C.c_int, C.POINTER(StageCfg),
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tmps_stage_destroy": (None, [C.c_void_p]),
    "tmps_stage_param_count": (C.c_int64, [C.c_void_p]),
    "tmps_stage_param_offset": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "tmps_stage_input_elems": (C.c_int64, [C.c_void_p]),
    "tmps_stage_output_elems": (C.c_int64, [C.c_void_p]),
    "tmps_stage_sync_params": (C.c_int, [C.c_void_p, C.c_void_p]),
    "tmps_stage_output_ptr": (C.c_void_p, [C.c_void_p, C.c_int]),
    "tmps_stage_version": (C.c_long, [C.c_void_p]),
    "tmps_stage_set_version": (C.c_int, [C.c_void_p, C.c_long]),
    "tmps_stage_use_graphs": (C.c_int, [C.c_void_p, C.c_int]),
    "tmps_stage_set_shadow": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]),
    "tmps_forward_micro_at": (C.c_int, [C.c_void_p, C.c_long, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p]),
    "tmps_schedule_shadow_versions": (C.c_int, [C.c_int, C.c_int, C.c_int]),
    "tmps_forward_micro": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tmps_forward_micro_static": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tmps_backward": (C.c_int, [C.c_void_p, C.POINTER(C.c_int), C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tmps_backward_at": (C.c_int, [C.c_void_p, C.c_long, C.POINTER(C.c_int), C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "tmps_schedule_plan_1f1b": (C.c_int, [C.c_int, C.c_int, C.POINTER(C.c_int32), C.c_size_t]),
    "tmps_schedule_run_1f1b": (C.c_int, [C.POINTER(C.c_void_p), C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                         C.POINTER(C.c_void_p), C.c_void_p, C.POINTER(C.c_int32)]),
    "tmps_update": (C.c_int, [C.c_void_p, C.c_void_p]),
    "tmps_schedule_plan": (C.c_int, [C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int32), C.c_size_t]),
    "tmps_schedule_stash_groups": (C.c_int, [C.c_int, C.c_int, C.c_int]),
    "tmps_version_diff_formula": (C.c_int, [C.c_int, C.c_int]),
    "tmps_version_diff_simulated": (C.c_int, [C.c_int, C.c_int]),
    "tmps_schedule_run": (C.c_int, [C.POINTER(C.c_void_p), C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                    C.POINTER(C.c_void_p), C.c_void_p, C.POINTER(C.c_int32)]),
    "tmps_schedule_run_vsync": (C.c_int, [C.POINTER(C.c_void_p), C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                          C.POINTER(C.c_void_p), C.c_void_p, C.POINTER(C.c_int32)]),
    "tmps_streams_create": (C.c_int, [C.POINTER(C.c_void_p), C.c_int]),
    "tmps_streams_destroy": (C.c_int, [C.POINTER(C.c_void_p), C.c_int]),
    "tmps_profile_enable": (C.c_int, [C.c_int]),
    "tmps_profile_read": (C.c_int, [C.POINTER(C.c_double), C.POINTER(C.c_int64), C.c_int]),
    "tmps_dense_gradients_joint": (C.c_int, [C.c_int, C.c_int64, C.c_int, C.c_int]),
    "tmps_pointwise_gradients_joint": (C.c_int, [C.c_int, C.c_int64, C.c_int, C.c_int]),
    "tmps_pool_affine_gradients_joint": (C.c_int, [C.c_int, C.c_int64, C.c_int, C.c_int, C.c_int]),
    "tmps_pointwise_forward_joint": (C.c_int, [C.c_int, C.c_int64, C.c_int, C.c_int]),
    "tmps_rotary": (C.c_int, [C.c_int, C.POINTER(RotaryDesc), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int64,
                              C.c_int, C.c_void_p]),
    "tmps_norm_join_forward": (C.c_int, [C.c_int, C.c_int, C.c_int64, C.c_int] + [C.c_void_p] * 10),
    "tmps_norm_join_workspace": (C.c_size_t, [C.c_int64, C.c_int]),
    "tmps_norm_join_backward": (C.c_int, [C.c_int, C.c_int, C.c_int64, C.c_int] + [C.c_void_p] * 14 + [C.c_size_t, C.c_void_p]),
    "tmps_distill_workspace": (C.c_size_t, [C.c_int64, C.c_int]),
    "tmps_distill": (C.c_int, [C.c_int, C.POINTER(DistillDesc), C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64,
                               C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tmps_short_conv_forward": (C.c_int, [C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int, C.c_void_p, C.c_int64] + [C.c_void_p] * 4 +
                                [C.c_int64, C.c_void_p, C.c_void_p]),
    "tmps_short_conv_workspace": (C.c_size_t, [C.c_int64, C.c_int64, C.c_int, C.c_int]),
    "tmps_short_conv_backward": (C.c_int, [C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64] +
                                 [C.c_void_p] * 5 + [C.c_int64] + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p]),
    "tmps_scan_workspace": (C.c_size_t, [C.POINTER(ScanDesc), C.c_int64, C.c_int64]),
    "tmps_scan_forward": (C.c_int, [C.c_int, C.POINTER(ScanDesc), C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64] + [C.c_void_p] * 5 +
                          [C.c_int64, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tmps_scan_backward_workspace": (C.c_size_t, [C.c_int, C.POINTER(ScanDesc), C.c_int64, C.c_int64]),
    "tmps_scan_backward": (C.c_int, [C.c_int, C.POINTER(ScanDesc), C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                     C.c_int64] + [C.c_void_p] * 5 + [C.c_int64, C.c_void_p, C.c_int64] + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p]),
    "tmps_group_norm_workspace": (C.c_size_t, [C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int, C.c_int]),
    "tmps_group_norm_forward": (C.c_int, [C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]),
    "tmps_group_norm_backward": (C.c_int, [C.c_int, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int] + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]),
    "tmps_clip_workspace": (C.c_size_t, [C.POINTER(Array), C.c_int]),
    "tmps_clip_gradients": (C.c_int, [C.POINTER(Array), C.c_int, C.c_float, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "tmps_last_error": (C.c_char_p, []),
}


def load_library():
    """Load libtmps.so and declare every exported symbol; raises if the library is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError("libtmps.so is not built (%s): run `python __graft_entry__.py`" % _LIB_PATH)
    lib_ = C.CDLL(_LIB_PATH)
    for name, (res, args) in EXPORTS.items():
        fn = getattr(lib_, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib_
    return _lib


def lib():
    return load_library()


def _check(rc):
    if rc < 0:
        raise TmpsError(rc, lib().tmps_last_error().decode())
    return rc


# ------------------------------------------------------------------------------- host-only calls
def schedule_plan(W, N, n_minibatches):
    n = _check(lib().tmps_schedule_plan(W, N, n_minibatches, None, 0))
    buf = (C.c_int32 * (7 * n))()
    _check(lib().tmps_schedule_plan(W, N, n_minibatches, buf, n))
    return np.frombuffer(buf, dtype=np.int32).reshape(n, 7).copy()


def schedule_plan_1f1b(W, n_batches):
    n = _check(lib().tmps_schedule_plan_1f1b(W, n_batches, None, 0))
    buf = (C.c_int32 * (7 * n))()
    _check(lib().tmps_schedule_plan_1f1b(W, n_batches, buf, n))
    return np.frombuffer(buf, dtype=np.int32).reshape(n, 7).copy()


def schedule_stash_groups(W, N, stage):
    return _check(lib().tmps_schedule_stash_groups(W, N, stage))


def schedule_shadow_versions(W, N, stage):
    return _check(lib().tmps_schedule_shadow_versions(W, N, stage))


def version_diff_formula(W, N):
    return _check(lib().tmps_version_diff_formula(W, N))


def version_diff_simulated(W, N):
    return _check(lib().tmps_version_diff_simulated(W, N))


KERNEL_CLASSES = ["dense_fwd", "dense_dgrad", "dense_wgrad", "conv_fwd", "conv_dgrad", "conv_wgrad", "softmax_ce",
                  "update", "pool_fwd", "pool_bwd", "relu_mask", "reduce", "copy", "event_pair", "splitk_finish", "slice_sum",
                  "layernorm", "attn_fwd", "attn_bwd", "embedding", "affine", "resadd", "dense_backward"]


def profile_enable(on):
    _check(lib().tmps_profile_enable(int(bool(on))))


def profile_read():
    """{class name: (total milliseconds, launches)} since the last read."""
    n = len(KERNEL_CLASSES)
    ms = (C.c_double * n)()
    cnt = (C.c_int64 * n)()
    _check(lib().tmps_profile_read(ms, cnt, n))
    return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNEL_CLASSES)}


def dense_gradients_joint(dtype, rows, din, dout):
    """Whether both gradients of a linear layer are one launch, timed under "dense_backward"."""
    return bool(lib().tmps_dense_gradients_joint(TMPS_BF16_F32MASTER if dtype == "bf16" else TMPS_F32, rows, din, dout))


def pointwise_gradients_joint(dtype, positions, cin, cout):
    """Whether the gradients of a 1 x 1 convolution and the affine layer behind it are one launch, timed under "affine"."""
    return bool(lib().tmps_pointwise_gradients_joint(TMPS_BF16_F32MASTER if dtype == "bf16" else TMPS_F32, positions, cin, cout))


def pool_affine_gradients_joint(dtype, positions, channels, window, stride):
    """Whether the gradient of max pooling and those of the affine layer below are one launch, timed under "pool_bwd"."""
    return bool(lib().tmps_pool_affine_gradients_joint(TMPS_BF16_F32MASTER if dtype == "bf16" else TMPS_F32, positions, channels, window, stride))


def pointwise_forward_joint(dtype, positions, cin, cout):
    """Whether a 1 x 1 convolution with its affine layer and a residual join is one launch with the convolution that reads the join first."""
    return bool(lib().tmps_pointwise_forward_joint(TMPS_BF16_F32MASTER if dtype == "bf16" else TMPS_F32, int(positions), cin, cout))


def _rotary_flags(interleaved, own_ladders):
    return (TMPS_FLAG_INTERLEAVED if interleaved else 0) | (TMPS_FLAG_OWN_LADDERS if own_ladders else 0)


def _float_bits(v):
    return int(np.float32(v).view(np.int32))


def distill_records(labels, ids, teacher):
    """The labels of a distillation layer: int32 [..., 1 + 2 k] from labels [...], a teacher's classes ids [..., k] and its logits [..., k]."""
    ids = np.asarray(ids, dtype=np.int32)
    bits = np.ascontiguousarray(np.asarray(teacher, dtype=np.float32)).view(np.int32)
    return np.concatenate([np.asarray(labels, dtype=np.int32)[..., None], ids, bits], axis=-1)


def layer_descs(specs):
    """Neutral layer dicts (workloads.configs) -> array of tmps_layer_desc."""
    arr = (LayerDesc * len(specs))()
    for d, sp in zip(arr, specs):
        k = sp["kind"]
        dims = [0] * 8
        if k == "linear":
            d.kind, dims[:4] = TMPS_LINEAR, [sp["din"], sp["dout"], sp.get("skip", 0), sp.get("rows", 1)]
            d.flags = TMPS_FLAG_RELU if sp["relu"] else (TMPS_FLAG_GELU if sp.get("act") == "gelu" else 0)
        elif k == "layernorm":
            if abs(sp["eps"] - 1e-5) > 1e-12:
                raise ValueError("the library's layer normalisation uses eps = 1e-5")
            d.kind, dims[:2] = TMPS_LAYERNORM, [sp["d"], sp["rows"]]
            d.flags = TMPS_FLAG_RMS if sp.get("rms") else 0
        elif k == "rotary":
            d.kind, dims[:8] = TMPS_ROTARY, [sp["s"], sp["d"], sp["heads"], sp["height"], sp["width"], sp["pairs_h"], sp["pairs_w"], sp["base"]]
            d.flags = _rotary_flags(sp["interleaved"], sp["own_ladders"])
        elif k == "norm_join":
            d.kind, dims[:3] = TMPS_NORMJOIN, [sp["d"], sp["rows"], sp["src"]]
            d.flags = _join_flags(sp["rms"], sp["gate"])
        elif k == "distill":
            d.kind, dims[:5] = TMPS_DISTILL, [sp["classes"], sp["rows"], sp["k"], _float_bits(sp["temperature"]), _float_bits(sp["alpha"])]
        elif k == "attention":
            d.kind, dims[:3] = TMPS_ATTENTION, [sp["s"], sp["d"], sp["heads"]]
        elif k == "embedding":
            d.kind, dims[:3] = TMPS_EMBEDDING, [sp["vocab"], sp["s"], sp["d"]]
        elif k == "conv":
            d.kind = TMPS_CONV2D
            dims[:8] = [sp["h"], sp["w"], sp["cin"], sp["cout"], sp["r"], sp["s"], sp["stride"], sp["pad"]]
            d.flags = (TMPS_FLAG_RELU if sp["relu"] else 0) | ((sp.get("src", 1) << 8) if sp.get("src", 1) > 1 else 0)
        elif k == "maxpool":
            d.kind, dims[:6] = TMPS_MAXPOOL, [sp["h"], sp["w"], sp["c"], sp["k"], sp["stride"], sp.get("pad", 0)]
        elif k == "affine":
            d.kind, dims[:3] = TMPS_AFFINE, [sp["h"], sp["w"], sp["c"]]
            d.flags = TMPS_FLAG_RELU if sp["relu"] else 0
        elif k == "resadd":
            d.kind, dims[:4] = TMPS_RESADD, [sp["h"], sp["w"], sp["c"], sp["src_b"]]
            d.flags = TMPS_FLAG_RELU if sp["relu"] else 0
        elif k == "avgpool":
            d.kind, dims[:3] = TMPS_AVGPOOL, [sp["h"], sp["w"], sp["c"]]
        elif k == "softmax_ce":
            d.kind, dims[:2] = TMPS_SOFTMAX_CE, [sp["classes"], sp.get("rows", 1)]
        else:
            raise ValueError("unknown layer kind %r" % k)
        for i, v in enumerate(dims):
            d.dims[i] = int(v)
    return arr


def stage_bytes(specs, cfg):
    out = [C.c_size_t() for _ in range(4)]
    descs = layer_descs(specs)
    _check(lib().tmps_stage_bytes(descs, len(specs), C.byref(cfg), *[C.byref(o) for o in out]))
    return tuple(o.value for o in out)


# ------------------------------------------------------------------------------------ operators on their own
# Gradients are calls as well (rotary's inverse, norm_join_backward, distill's second result): nothing is recorded for torch's backward pass, and tensors that ask for it are refused
# outside of torch.no_grad().
def _torch():
    global _torch_of, _raw_stream, _current_device
    if _torch_of is None:
        import torch
        _raw_stream, _current_device = _short_ways(torch, torch._C)
        _torch_of = torch
    return _torch_of


def _short_ways(torch, private):
    """(a GPU's index -> its current stream's handle, () -> the current GPU's index).  The private ones, where this torch has them, make no object (0.1 us instead of 1.9) and ask
    less (a process that has tensors on a GPU has initialised it)."""
    return (getattr(private, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream),
            getattr(private, "_cuda_getDevice", None) or torch.cuda.current_device)


_torch_of = _raw_stream = _current_device = None


def _dtype_code(t):
    torch = _torch()
    if t.dtype is torch.float32:
        return TMPS_F32
    if t.dtype is torch.bfloat16:
        return TMPS_BF16_F32MASTER
    raise ValueError("%s: the library computes in float32 and bfloat16" % t.dtype)


def _unrecorded(name, t):
    if t.requires_grad and _torch().is_grad_enabled():
        raise ValueError("%s asks for a gradient, which is a call of its own here and not recorded: call with detached tensors or under torch.no_grad()" % name)


def _operand(name, t, shape, dtype, device):
    """A tensor's address, after a check of what it is (rows contiguous); None stays None."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.device == device:
        if t.requires_grad:
            _unrecorded(name, t)
        return t.data_ptr()
    raise ValueError("%s: a contiguous %s tensor of shape %s on %s is wanted, not %s %s on %s"
                     % (name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))


def _within(stream, device):
    """`stream` (a stream, or its handle) as the current one: what a call allocates there, its results and workspaces, then belongs to the stream that uses it."""
    cuda = _torch().cuda
    if device.type != "cuda":
        raise ValueError("tensors on a GPU are wanted, not on %s" % device)
    if not hasattr(stream, "cuda_stream"):
        stream = cuda.ExternalStream(int(stream), device=device) if int(stream) else cuda.default_stream(device)
    if stream.device != device:
        raise ValueError("stream: one of %s is wanted, not of %s" % (device, stream.device))
    return cuda.stream(stream)


def _call(fn, device, stream, *args):
    """fn(..., stream) on a GPU's current stream, with that GPU current.  stream is None: another stream is made the current one (_within) before results and workspaces are
    allocated, which belong to the stream that is current then."""
    torch = _torch()
    if device.type != "cuda":
        raise ValueError("tensors on a GPU are wanted, not on %s" % device)
    if stream is not None:
        raise ValueError("a call runs on the current stream")
    index = device.index
    handle = _raw_stream(index)
    if index == _current_device():
        rc = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, handle)
    if rc < 0:
        _check(rc)


def rotary(x, positions, heads, dh, pairs, base=10000.0, interleaved=False, own_ladders=False, inverse=False, out=None, stream=None):
    """Rotary positions (tmps_rotary) of the `heads` heads of dh features that begin each row of x [rows, features]: pairs = (time, height, width)
    pairs of features that turn with each axis of positions, int32 [n, 3], which the rows take in turn.  inverse: back, the gradient's way.
    out (default: a new tensor [rows, heads * dh]) may be x, or a view of rows of its own stride.  Returns out.  On the current stream, or on `stream`, which a new tensor then
    belongs to; it waits for no other.  A tensor that asks for a gradient is refused while gradients are recorded (all of these calls do so)."""
    if stream is not None:
        with _within(stream, x.device):
            return rotary(x, positions, heads, dh, pairs, base, interleaved, own_ladders, inverse, out)
    torch = _torch()
    code, width = _dtype_code(x), heads * dh
    if x.dim() != 2 or x.shape[1] < width or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("x: rows of at least %d neighbouring features are wanted, not shape %s, strides %s" % (width, tuple(x.shape), x.stride()))
    if positions.dim() != 2 or positions.shape[1] != 3:
        raise ValueError("positions: [n, 3] is wanted, not %s" % (tuple(positions.shape),))
    if len(pairs) != 3:
        raise ValueError("pairs: a number for each of three axes is wanted")
    rows = x.shape[0]
    pos = _operand("positions", positions, positions.shape, torch.int32, x.device)
    out_stride = width
    if out is None:
        out = torch.empty(rows, width, dtype=x.dtype, device=x.device)
    elif out.dim() != 2 or out.shape[0] != rows or out.shape[1] < width or (out.shape[1] > 1 and out.stride(1) != 1) or out.dtype != x.dtype or out.device != x.device:
        raise ValueError("out: %d rows of at least %d neighbouring %s features on %s are wanted" % (rows, width, x.dtype, x.device))
    else:
        out_stride = out.stride(0)
    if x.requires_grad or out.requires_grad:
        _unrecorded("x" if x.requires_grad else "out", x if x.requires_grad else out)
    d = RotaryDesc(heads, dh, Axes(*pairs), _rotary_flags(interleaved, own_ladders), base)
    _call(load_library().tmps_rotary, x.device, None, code, C.byref(d), x.data_ptr(), x.stride(0), out.data_ptr(), out_stride, pos, positions.shape[0], rows, int(inverse))
    return out


def _join_flags(rms, gate):
    return (TMPS_FLAG_RMS if rms else 0) | (TMPS_FLAG_GATE if gate else 0)


def norm_join(x, r, gain, scale, pre_gain=None, pre_shift=None, rms=False, gate=False, y=None, u=None, stats=None, stream=None):
    """y = scale r + g gain n(f), u = n(y) pre_gain + pre_shift over rows of r [rows, D] (tmps_norm_join_forward): x holds f, with `gate` rows [f | a] with
    g = 1 / (1 + exp(-a)); n is layer normalisation, with `rms` without its mean (then without pre_shift); without pre_gain u is None.  Returns
    (y, u, stats); y may be given as r.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, r.device):
            return norm_join(x, r, gain, scale, pre_gain, pre_shift, rms, gate, y, u, stats)
    torch = _torch()
    code = _dtype_code(r)
    if r.dim() != 2:
        raise ValueError("r: [rows, features] is wanted, not %s" % (tuple(r.shape),))
    (rows, D), t, dev, f32 = r.shape, r.dtype, r.device, torch.float32
    # (what is allocated here needs no check)
    if y is None:
        y = torch.empty(rows, D, dtype=t, device=dev)
        to_y = y.data_ptr()
    else:
        to_y = _operand("y", y, (rows, D), t, dev)
    if u is None and pre_gain is not None:
        u = torch.empty(rows, D, dtype=t, device=dev)
        to_u = u.data_ptr()
    else:
        to_u = _operand("u", u, (rows, D), t, dev)
    if stats is None:
        stats = torch.empty(rows, 4, dtype=f32, device=dev)
        to_stats = stats.data_ptr()
    else:
        to_stats = _operand("stats", stats, (rows, 4), f32, dev)
    _call(load_library().tmps_norm_join_forward, dev, None, code, _join_flags(rms, gate), rows, D, _operand("x", x, (rows, 2 * D if gate else D), t, dev),
          _operand("r", r, (rows, D), t, dev), _operand("gain", gain, (D,), f32, dev), _operand("scale", scale, (D,), f32, dev), to_y,
          _operand("pre_gain", pre_gain, (D,), f32, dev), _operand("pre_shift", pre_shift, (D,), f32, dev), to_u, to_stats)
    return y, u, stats


def norm_join_backward(dy, du, x, r, y, stats, gain, scale, pre_gain=None, rms=False, gate=False, dx=None, dr=None, stream=None):
    """Gradients of norm_join from dy and du (one of them may be None; with du also y and pre_gain are needed): (dx, dr, dgain, dscale, dpre_gain,
    dpre_shift), those of parameters fp32, the last two None without du, the last with `rms`.  dr may be given as dy.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, r.device):
            return norm_join_backward(dy, du, x, r, y, stats, gain, scale, pre_gain, rms, gate, dx, dr)
    torch = _torch()
    code = _dtype_code(r)
    if r.dim() != 2:
        raise ValueError("r: [rows, features] is wanted, not %s" % (tuple(r.shape),))
    (rows, D), t, dev = r.shape, r.dtype, r.device
    wide = 2 * D if gate else D
    if dx is None:
        dx = torch.empty(rows, wide, dtype=t, device=dev)
        to_dx = dx.data_ptr()
    else:
        to_dx = _operand("dx", dx, (rows, wide), t, dev)
    if dr is None:
        dr = torch.empty(rows, D, dtype=t, device=dev)
        to_dr = dr.data_ptr()
    else:
        to_dr = _operand("dr", dr, (rows, D), t, dev)
    grads = torch.empty(4, D, dtype=torch.float32, device=dev)
    need = load_library().tmps_norm_join_workspace(rows, D)
    ws = torch.empty(max(need, 4), dtype=torch.uint8, device=dev)
    at = grads.data_ptr()
    _call(load_library().tmps_norm_join_backward, dev, None, code, _join_flags(rms, gate), rows, D, _operand("dy", dy, (rows, D), t, dev), _operand("du", du, (rows, D), t, dev),
          _operand("x", x, (rows, wide), t, dev), _operand("r", r, (rows, D), t, dev), _operand("y", y, (rows, D), t, dev),
          _operand("stats", stats, (rows, 4), torch.float32, dev), _operand("gain", gain, (D,), torch.float32, dev),
          _operand("scale", scale, (D,), torch.float32, dev), _operand("pre_gain", pre_gain, (D,), torch.float32, dev), to_dx, to_dr, at, at + 8 * D if du is not None else None, ws.data_ptr(), need)
    dgain, dscale, dpre_gain, dpre_shift = grads.unbind(0)
    if du is None:
        return dx, dr, dgain, dscale, None, None
    return dx, dr, dgain, dscale, dpre_gain, None if rms else dpre_shift


def distill(logits, labels, ids, teacher, temperature=1.0, alpha=1.0, grad_scale=None, dtype="f32", gradient=True, stream=None):
    """Distillation loss of each row of fp32 logits [rows, classes] against a teacher's logits [rows, k] of the classes ids (int32 [rows, k], -1: no entry)
    and labels (int32 [rows], -1: none; may be None), with its gradient times grad_scale (default: 1 / rows, for the mean) in `dtype` (tmps_distill).
    Returns (row_loss, dlogits); dlogits is None without `gradient`.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, logits.device):
            return distill(logits, labels, ids, teacher, temperature, alpha, grad_scale, dtype, gradient)
    torch = _torch()
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits: [rows, classes], ids: [rows, k] are wanted")
    if dtype not in ("f32", "bf16"):
        raise ValueError("dtype: \"f32\" or \"bf16\"")
    (rows, classes), k, dev = logits.shape, ids.shape[1], logits.device
    row_loss = torch.empty(rows, dtype=torch.float32, device=dev)
    dlogits = torch.empty(rows, classes, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=dev) if gradient else None
    d = DistillDesc(classes, k, temperature, alpha, 1.0 / max(rows, 1) if grad_scale is None else grad_scale)
    need = load_library().tmps_distill_workspace(rows, classes)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(load_library().tmps_distill, dev, None, TMPS_BF16_F32MASTER if dtype == "bf16" else TMPS_F32, C.byref(d), rows,
          _operand("logits", logits, (rows, classes), torch.float32, dev), _operand("labels", labels, (rows,), torch.int32, dev), 1,
          _operand("ids", ids, (rows, k), torch.int32, dev), _operand("teacher", teacher, (rows, k), torch.float32, dev), k,
          dlogits.data_ptr() if gradient else None, row_loss.data_ptr(), ws.data_ptr() if need else None, need)
    return row_loss, dlogits


def _rows_of(name, t, width, dtype, device, rows=None):
    """(address, stride) of rows of `width` neighbouring elements, which may be columns of wider rows."""
    if t.dim() != 2 or t.shape[1] != width or (rows is not None and t.shape[0] != rows) or t.dtype is not dtype or t.device != device or \
            (width > 1 and t.stride(1) != 1 and t.shape[0] > 0):
        raise ValueError("%s: %s rows of %d neighbouring %s elements on %s are wanted, not %s %s of strides %s on %s"
                         % (name, "some" if rows is None else rows, width, dtype, device, t.dtype, tuple(t.shape), t.stride(), t.device))
    if t.requires_grad:
        _unrecorded(name, t)
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else width


def _new_rows(name, t, rows, width, dtype, device):
    """(tensor, address, stride) of a result's rows: those given, or new ones."""
    if t is None:
        t = _torch().empty(rows, width, dtype=dtype, device=device)
        return t, t.data_ptr(), width
    return (t,) + _rows_of(name, t, width, dtype, device, rows)


def _samples(rows, positions):
    if positions < 1 or rows % positions:
        raise ValueError("positions: rows are samples of as many positions each, not %d rows of %d" % (rows, positions))
    return rows // positions


def _workspace(need, device):
    return _torch().empty(max(need, 16), dtype=_torch().uint8, device=device) if need else None


def short_conv(x, weight, bias=None, positions=1, tail=None, want_tail=False, silu=True, out=None, tail_out=None, stream=None):
    """A causal convolution along the positions of each sample, channels apart, with SiLU behind it (tmps_short_conv_forward): x [samples * positions, channels] (rows may
    be columns of wider rows), weight fp32 [channels, taps], bias fp32 [channels] or None, tail [samples, taps - 1, channels]: the inputs before the first
    position (None: zeros).  Returns (y, tail): the last taps - 1 inputs, None unless want_tail or a tensor tail_out for them is given (for one position it may be
    tail).  out may be columns of wider rows.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, x.device):
            return short_conv(x, weight, bias, positions, tail, want_tail, silu, out, tail_out)
    torch = _torch()
    code, t, dev = _dtype_code(x), x.dtype, x.device
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x: [rows, channels], weight: [channels, taps] are wanted")
    (rows, channels), taps = x.shape, weight.shape[1]
    samples = _samples(rows, positions)
    at_x, x_stride = _rows_of("x", x, channels, t, dev)
    out, at_y, y_stride = _new_rows("out", out, rows, channels, t, dev)
    if tail_out is None and want_tail:
        tail_out = torch.empty(samples, taps - 1, channels, dtype=t, device=dev)
    _call(load_library().tmps_short_conv_forward, dev, None, code, TMPS_FLAG_SILU if silu else 0, samples, positions, channels, taps, at_x, x_stride,
          _operand("weight", weight, (channels, taps), torch.float32, dev), _operand("bias", bias, (channels,), torch.float32, dev),
          _operand("tail", tail, (samples, taps - 1, channels), t, dev), at_y, y_stride, _operand("tail_out", tail_out, (samples, taps - 1, channels), t, dev))
    return out, tail_out


def short_conv_backward(dy, x, weight, bias=None, positions=1, tail=None, dtail=None, silu=True, dx=None, stream=None):
    """Gradients of short_conv from dy and, w.r.t. the tail it returned, dtail (None: none): (dx, dweight, dbias, dtail_in), those of parameters fp32, dbias None without a
    bias, dtail_in None without a tail.  dy, x and dx may be columns of wider rows.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, x.device):
            return short_conv_backward(dy, x, weight, bias, positions, tail, dtail, silu, dx)
    torch = _torch()
    code, t, dev, f32 = _dtype_code(x), x.dtype, x.device, torch.float32
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x: [rows, channels], weight: [channels, taps] are wanted")
    (rows, channels), taps = x.shape, weight.shape[1]
    samples = _samples(rows, positions)
    at_x, x_stride = _rows_of("x", x, channels, t, dev)
    at_dy, dy_stride = _rows_of("dy", dy, channels, t, dev, rows)
    dx, at_dx, dx_stride = _new_rows("dx", dx, rows, channels, t, dev)
    dtail_in = torch.empty(samples, taps - 1, channels, dtype=t, device=dev) if tail is not None else None
    grads = torch.empty(channels * (taps + (bias is not None)), dtype=f32, device=dev)
    need = load_library().tmps_short_conv_workspace(samples, positions, channels, taps)
    ws = _workspace(need, dev)
    _call(load_library().tmps_short_conv_backward, dev, None, code, TMPS_FLAG_SILU if silu else 0, samples, positions, channels, taps, at_dy, dy_stride, at_x, x_stride,
          _operand("weight", weight, (channels, taps), f32, dev), _operand("bias", bias, (channels,), f32, dev),
          _operand("tail", tail, (samples, taps - 1, channels), t, dev), _operand("dtail", dtail, (samples, taps - 1, channels), t, dev), at_dx, dx_stride,
          dtail_in.data_ptr() if dtail_in is not None else None, grads.data_ptr(), ws.data_ptr() if need else None, need)
    return dx, grads[:channels * taps].view(channels, taps), grads[channels * taps:] if bias is not None else None, dtail_in


def _scan_shape(x, a_log, positions, groups, state_features):
    if x.dim() != 2 or a_log.dim() != 1:
        raise ValueError("x: [rows, features], a_log: [heads] are wanted")
    (rows, wide), heads = x.shape, a_log.shape[0]
    inner = wide - 2 * groups * state_features
    if groups < 1 or state_features < 1 or heads < 1 or inner < 1 or inner % heads:
        raise ValueError("x: rows [x (heads * features) | B (groups * state_features) | C (groups * state_features)] are wanted, not %d features for %d heads, "
                         "%d groups and %d state_features" % (wide, heads, groups, state_features))
    return rows, wide, heads, inner, _samples(rows, positions), ScanDesc(heads, inner // heads, groups, state_features)


def selective_scan(x, dt, a_log, skip, dt_bias, positions, state_features, groups=1, state=None, want_state=False, out=None, state_out=None, stream=None):
    """A selective state space (tmps_scan_forward): per head and position delta = softplus(dt + dt_bias), S <- exp(-delta exp(a_log)) S + delta x B', y = S C + skip x.
    x: rows [x (heads * features) | B (groups * state_features) | C (groups * state_features)], dt: rows [heads] (both may be columns of wider rows), samples of
    `positions` rows each; a_log, skip, dt_bias fp32 [heads]; state fp32 [samples, heads, features, state_features] before the first position (None: zeros).
    Returns (y, state): y [rows, heads * features] (out, where given, may be columns of wider rows) and the state behind the last position, None unless want_state
    or a tensor state_out for it is given, which may be state.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, x.device):
            return selective_scan(x, dt, a_log, skip, dt_bias, positions, state_features, groups, state, want_state, out, state_out)
    torch = _torch()
    code, t, dev, f32 = _dtype_code(x), x.dtype, x.device, torch.float32
    rows, wide, heads, inner, samples, d = _scan_shape(x, a_log, positions, groups, state_features)
    of_state = (samples, heads, inner // heads, state_features)
    at_x, x_stride = _rows_of("x", x, wide, t, dev)
    at_dt, dt_stride = _rows_of("dt", dt, heads, t, dev, rows)
    out, at_y, y_stride = _new_rows("out", out, rows, inner, t, dev)
    if state_out is None and want_state:
        state_out = torch.empty(of_state, dtype=f32, device=dev)
    need = load_library().tmps_scan_workspace(C.byref(d), samples, positions)
    ws = _workspace(need, dev)
    _call(load_library().tmps_scan_forward, dev, None, code, C.byref(d), samples, positions, at_x, x_stride, at_dt, dt_stride,
          _operand("a_log", a_log, (heads,), f32, dev), _operand("skip", skip, (heads,), f32, dev), _operand("dt_bias", dt_bias, (heads,), f32, dev),
          _operand("state", state, of_state, f32, dev), at_y, y_stride, _operand("state_out", state_out, of_state, f32, dev), ws.data_ptr() if need else None, need)
    return out, state_out


def selective_scan_backward(dy, x, dt, a_log, skip, dt_bias, positions, state_features, groups=1, state=None, dstate=None, dx=None, ddt=None, stream=None):
    """Gradients of selective_scan from dy and, w.r.t. the state it returned, dstate (None: none): (dx, ddt, da_log, dskip, ddt_bias, dstate_in), dx rows as x's,
    those of parameters and of the state fp32, dstate_in None without a state.  dx and ddt, where given, may be columns of wider rows.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, x.device):
            return selective_scan_backward(dy, x, dt, a_log, skip, dt_bias, positions, state_features, groups, state, dstate, dx, ddt)
    torch = _torch()
    code, t, dev, f32 = _dtype_code(x), x.dtype, x.device, torch.float32
    rows, wide, heads, inner, samples, d = _scan_shape(x, a_log, positions, groups, state_features)
    of_state = (samples, heads, inner // heads, state_features)
    at_dy, dy_stride = _rows_of("dy", dy, inner, t, dev, rows)
    at_x, x_stride = _rows_of("x", x, wide, t, dev)
    at_dt, dt_stride = _rows_of("dt", dt, heads, t, dev, rows)
    dx, at_dx, dx_stride = _new_rows("dx", dx, rows, wide, t, dev)
    ddt, at_ddt, ddt_stride = _new_rows("ddt", ddt, rows, heads, t, dev)
    dstate_in = torch.empty(of_state, dtype=f32, device=dev) if state is not None else None
    grads = torch.empty(3, heads, dtype=f32, device=dev)
    need = load_library().tmps_scan_backward_workspace(code, C.byref(d), samples, positions)
    ws = _workspace(need, dev)
    _call(load_library().tmps_scan_backward, dev, None, code, C.byref(d), samples, positions, at_dy, dy_stride, _operand("dstate", dstate, of_state, f32, dev), at_x, x_stride,
          at_dt, dt_stride, _operand("a_log", a_log, (heads,), f32, dev), _operand("skip", skip, (heads,), f32, dev), _operand("dt_bias", dt_bias, (heads,), f32, dev),
          _operand("state", state, of_state, f32, dev), at_dx, dx_stride, at_ddt, ddt_stride, grads.data_ptr(),
          dstate_in.data_ptr() if dstate_in is not None else None, ws.data_ptr() if need else None, need)
    return (dx, ddt) + tuple(grads.unbind(0)) + (dstate_in,)


def _act_flags(act, rms):
    acts = {None: 0, "relu": TMPS_FLAG_RELU, "gelu": TMPS_FLAG_GELU, "silu": TMPS_FLAG_SILU}
    if act not in acts:
        raise ValueError('act: None, "relu", "gelu" or "silu"')
    return acts[act] | (TMPS_FLAG_RMS if rms else 0)


def group_norm(x, gain, shift=None, groups=1, positions=1, act=None, rms=False, y=None, stats=None, stream=None):
    """Group norm of maps [samples * positions, channels], channels last, and the activation behind it (tmps_group_norm_forward): y = act(gain xhat + shift), xhat = (x - mean) /
    sqrt(var + 1e-5) over a sample's positions and the channels / groups channels of a group, with `rms` x / sqrt(mean(x^2) + 1e-5); act: None, "relu", "gelu" or
    "silu"; shift may be None.  Returns (y, stats): stats fp32 [samples, groups, 2], mean and 1/std.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, x.device):
            return group_norm(x, gain, shift, groups, positions, act, rms, y, stats)
    torch = _torch()
    code, t, dev, f32 = _dtype_code(x), x.dtype, x.device, torch.float32
    if x.dim() != 2:
        raise ValueError("x: [rows, channels] is wanted, not %s" % (tuple(x.shape),))
    rows, channels = x.shape
    samples = _samples(rows, positions)
    if y is None:
        y = torch.empty(rows, channels, dtype=t, device=dev)
    if stats is None:
        stats = torch.empty(samples, max(groups, 0), 2, dtype=f32, device=dev)
    need = load_library().tmps_group_norm_workspace(code, samples, positions, channels, groups, 0)
    ws = _workspace(need, dev)
    _call(load_library().tmps_group_norm_forward, dev, None, code, _act_flags(act, rms), samples, positions, channels, groups, _operand("x", x, (rows, channels), t, dev),
          _operand("gain", gain, (channels,), f32, dev), _operand("shift", shift, (channels,), f32, dev), _operand("y", y, (rows, channels), t, dev),
          _operand("stats", stats, (samples, groups, 2), f32, dev), ws.data_ptr() if need else None, need)
    return y, stats


def group_norm_backward(dy, x, stats, gain, shift=None, groups=1, positions=1, act=None, rms=False, dx=None, stream=None):
    """Gradients of group_norm from dy and the stats that it returned: (dx, dgain, dshift), those of parameters fp32, dshift None without a shift.  `stream` as for rotary."""
    if stream is not None:
        with _within(stream, x.device):
            return group_norm_backward(dy, x, stats, gain, shift, groups, positions, act, rms, dx)
    torch = _torch()
    code, t, dev, f32 = _dtype_code(x), x.dtype, x.device, torch.float32
    if x.dim() != 2:
        raise ValueError("x: [rows, channels] is wanted, not %s" % (tuple(x.shape),))
    rows, channels = x.shape
    samples = _samples(rows, positions)
    if dx is None:
        dx = torch.empty(rows, channels, dtype=t, device=dev)
    grads = torch.empty(2, channels, dtype=f32, device=dev)
    need = load_library().tmps_group_norm_workspace(code, samples, positions, channels, groups, 1)
    ws = _workspace(need, dev)
    _call(load_library().tmps_group_norm_backward, dev, None, code, _act_flags(act, rms), samples, positions, channels, groups, _operand("dy", dy, (rows, channels), t, dev),
          _operand("x", x, (rows, channels), t, dev), _operand("stats", stats, (samples, groups, 2), f32, dev), _operand("gain", gain, (channels,), f32, dev),
          _operand("shift", shift, (channels,), f32, dev), _operand("dx", dx, (rows, channels), t, dev), grads.data_ptr(), ws.data_ptr() if need else None, need)
    dgain, dshift = grads.unbind(0)
    return dx, dgain, dshift if shift is not None else None


_DTYPE_OF, _REQUIRES_GRAD_OF = operator.attrgetter("dtype"), operator.attrgetter("requires_grad")


def clip_gradients(grads, limit, out=None, stream=None):
    """The norm of all tensors of `grads` together, fp32 of no dimension, and each of them times limit / norm where that is less than one, in place or in the tensors `out`,
    of the same types and numbers of elements (tmps_clip_gradients).  limit = inf: the norm alone.  A norm that is not finite (in fp32) leaves the values as they are.  Tensors are
    contiguous, fp32 or bf16.  `stream` as for rotary."""
    grads = list(grads)
    if not grads:
        raise ValueError("grads: one tensor at least is wanted")
    dev = grads[0].device
    if stream is not None:
        with _within(stream, dev):
            return clip_gradients(grads, limit, out)
    torch = _torch()
    to = grads if out is None else list(out)
    if len(to) != len(grads):
        raise ValueError("out: %d tensors are wanted, not %d" % (len(grads), len(to)))
    if dev.type != "cuda":
        raise ValueError("tensors on a GPU are wanted, not on %s" % dev)
    # (a few attributes of each of hundreds of tensors: they are what such a call costs the host)
    many, n, T = grads if out is None else grads + to, len(grads), torch.Tensor
    types, sizes = list(map(_DTYPE_OF, many)), list(map(T.numel, many))
    kinds = list(map({torch.float32: TMPS_F32, torch.bfloat16: TMPS_BF16_F32MASTER}.get, types[:n]))
    if None in kinds:
        _dtype_code(grads[kinds.index(None)])
    if set(map(T.get_device, many)) != {dev.index} or not all(map(T.is_contiguous, many)) or any(map(_REQUIRES_GRAD_OF, many)):
        for k, g in enumerate(many):
            _operand("grads" if k < n else "out", g, g.shape, g.dtype, dev)
    if out is not None and (types[n:] != types[:n] or sizes[n:] != sizes[:n]):
        raise ValueError("out: tensors of the types and sizes of grads are wanted")
    record = np.empty(n, dtype=_ARRAY)
    at = list(map(T.data_ptr, many))
    record["data"], record["n"], record["dtype"] = at[:n], sizes[:n], kinds
    record["out"] = at[n:] if out is not None else 0 if limit == float("inf") else at
    arrays = C.cast(record.ctypes.data, C.POINTER(Array))
    norm = torch.empty((), dtype=torch.float32, device=dev)
    need = load_library().tmps_clip_workspace(arrays, len(grads))
    ws = _workspace(need, dev)
    _call(load_library().tmps_clip_gradients, dev, None, arrays, len(grads), limit, norm.data_ptr(), ws.data_ptr() if need else None, need)
    return norm


# ------------------------------------------------------------------------------------ device side
class Stage:
    """One pipeline worker on a GPU.  Owns the four device regions (torch tensors) the library works in."""

    def __init__(self, specs, dtype, micro_batch, n_micro, max_stash, lr, momentum, borrow_input=False,
                 device="cuda:0"):
        import torch
        self.torch = torch
        self.logical_specs = list(specs)
        # bf16 contractions fetch 8 channels per 16-byte load: a stage that starts with a convolution on
        # fewer channels (an RGB image) is handed channel-padded inputs and filters (zeros), which leaves
        # every result unchanged; set_params / get_* / prepare_input / crop_input_grad convert.
        self.cin, self.cin_pad = None, None
        specs = list(specs)
        if dtype == "bf16" and specs[0]["kind"] == "conv" and specs[0]["cin"] % 8 != 0:
            self.cin = specs[0]["cin"]
            self.cin_pad = (self.cin + 7) // 8 * 8
            specs[0] = dict(specs[0], cin=self.cin_pad)
        self.specs = specs
        self.device = torch.device(device)
        self.is_last = specs[-1]["kind"] in ("softmax_ce", "distill")
        self.cfg = StageCfg(TMPS_BF16_F32MASTER if dtype == "bf16" else TMPS_F32, micro_batch, n_micro, max_stash,
                            int(self.is_last), int(borrow_input), lr, momentum)
        self.act_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.descs = layer_descs(specs)
        sizes = stage_bytes(specs, self.cfg)
        # (nothing in the scratch region is read before a kernel has written it)
        self.regions = [torch.zeros(max(s, 256), dtype=torch.uint8, device=self.device) for s in sizes[:3]]
        self.regions.append(torch.empty(max(sizes[3], 256), dtype=torch.uint8, device=self.device))
        h = C.c_void_p()
        _check(lib().tmps_stage_create(C.byref(h), self.descs, len(specs), C.byref(self.cfg),
                                       *[C.c_void_p(r.data_ptr()) for r in self.regions]))
        self.handle = h
        self.P = lib().tmps_stage_param_count(h)
        self.in_elems = lib().tmps_stage_input_elems(h)
        self.out_elems = lib().tmps_stage_output_elems(h)
        self.micro, self.N = micro_batch, n_micro

    def __del__(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.tmps_stage_destroy(self.handle)
            self.handle = None

    # flat fp32 views into the device regions
    def _flat(self, region, index):
        t = self.regions[region][index * self.P * 4:(index + 1) * self.P * 4]
        return t.view(self.torch.float32)

    def param_offset(self, layer, which):
        off, cnt = C.c_int64(), C.c_int64()
        _check(lib().tmps_stage_param_offset(self.handle, layer, which, C.byref(off), C.byref(cnt)))
        return off.value, cnt.value

    def _get(self, flat):
        host = flat.cpu().numpy()
        out = []
        for li, sp in enumerate(self.specs):
            p = {}
            for which, key in ((0, "w"), (1, "b")):
                off, cnt = self.param_offset(li, which)
                if cnt:
                    p[key] = host[off:off + cnt].copy()
            if "w" in p:
                if sp["kind"] == "linear":
                    p["w"] = p["w"].reshape(sp["dout"], sp["din"])
                elif sp["kind"] == "conv":
                    p["w"] = p["w"].reshape(sp["cout"], sp["r"], sp["s"], sp["cin"])
                    if li == 0 and self.cin_pad:
                        p["w"] = np.ascontiguousarray(p["w"][..., :self.cin])
                elif sp["kind"] == "embedding":
                    p["w"] = p["w"].reshape(sp["vocab"], sp["d"])
                    p["b"] = p["b"].reshape(sp["s"], sp["d"])
            out.append(p)
        return out

    def set_params(self, params, stream=None):
        """Write fp32 master parameters (per layer dicts with 'w', 'b'), clear momentum, refresh the working copy."""
        torch = self.torch
        host = np.zeros(self.P, dtype=np.float32)
        for li, p in enumerate(params):
            for which, key in ((0, "w"), (1, "b")):
                off, cnt = self.param_offset(li, which)
                if cnt:
                    v = np.asarray(p[key], dtype=np.float32)
                    if li == 0 and key == "w" and self.cin_pad:
                        v = np.concatenate([v, np.zeros(v.shape[:-1] + (self.cin_pad - self.cin,), np.float32)], axis=-1)
                    host[off:off + cnt] = v.reshape(-1)
        self._flat(0, 0).copy_(torch.from_numpy(host))
        self.regions[1].zero_()
        torch.cuda.synchronize(self.device)
        _check(lib().tmps_stage_sync_params(self.handle, C.c_void_p(self._stream(stream))))
        torch.cuda.synchronize(self.device)

    def prepare_input(self, x):
        """Host array [rows, ...] -> device tensor in the layout and dtype the stage reads."""
        torch = self.torch
        if self.specs[0]["kind"] == "embedding":
            return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=np.int32))).to(self.device)
        x = np.asarray(x, dtype=np.float32)
        if self.cin_pad:
            x = np.concatenate([x, np.zeros(x.shape[:-1] + (self.cin_pad - self.cin,), np.float32)], axis=-1)
        return torch.from_numpy(np.ascontiguousarray(x)).to(self.act_dtype).to(self.device)

    def crop_input_grad(self, dx, rows):
        """Device gradient w.r.t. the stage input -> host fp32 array with the logical channel count."""
        a = dx.float().cpu().numpy().reshape(rows, -1)
        if self.cin_pad:
            a = a.reshape(-1, self.cin_pad)[:, :self.cin].reshape(rows, -1)
        return a

    def get_params(self):
        return self._get(self._flat(0, 0))

    def get_grads(self):
        return self._get(self._flat(1, 1))

    def get_momentum(self):
        return self._get(self._flat(1, 0))

    def _stream(self, stream):
        if stream is None:
            return self.torch.cuda.current_stream(self.device).cuda_stream
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def version(self):
        return lib().tmps_stage_version(self.handle)

    def set_shadow(self, n_versions):
        """Vertical weight stashing: keep the parameters of the last n_versions updates (a device region of its own)."""
        torch = self.torch
        one = self.regions[0].numel()
        self.shadow = torch.zeros(max(one * n_versions, 256), dtype=torch.uint8, device=self.device) if n_versions else None
        _check(lib().tmps_stage_set_shadow(self.handle, C.c_void_p(self.shadow.data_ptr()) if n_versions else None,
                                           one * n_versions, n_versions))

    def forward_micro_at(self, version, slot, x, y=None, labels=None, loss_out=None, stream=None):
        _check(lib().tmps_forward_micro_at(
            self.handle, version, slot, C.c_void_p(x.data_ptr()), C.c_void_p(y.data_ptr()) if y is not None else None,
            C.c_void_p(labels.data_ptr()) if labels is not None else None,
            C.c_void_p(loss_out.data_ptr()) if loss_out is not None else None, C.c_void_p(self._stream(stream))))

    # ---- stage-wise checkpoints (section "Checkpointing") ----
    def save_checkpoint(self, directory, stage_index, epoch):
        """Write this stage's master parameters, momentum and version to its own file (no other stage is involved)."""
        from . import checkpoint
        self.torch.cuda.synchronize(self.device)
        return checkpoint.write_stage(directory, stage_index, epoch, self.version(), self._flat(0, 0).cpu().numpy(),
                                      self._flat(1, 0).cpu().numpy())

    def load_checkpoint(self, directory, stage_index, epoch, stream=None):
        from . import checkpoint
        torch = self.torch
        ck = checkpoint.read_stage(directory, stage_index, epoch)
        if ck["params"].size != self.P:
            raise checkpoint.CheckpointError("stage %d: %d parameters in the file, %d in the stage"
                                             % (stage_index, ck["params"].size, self.P))
        self._flat(0, 0).copy_(torch.from_numpy(ck["params"]))
        self._flat(1, 0).copy_(torch.from_numpy(ck["momentum"]))
        torch.cuda.synchronize(self.device)
        _check(lib().tmps_stage_sync_params(self.handle, C.c_void_p(self._stream(stream))))
        _check(lib().tmps_stage_set_version(self.handle, int(ck["version"])))
        torch.cuda.synchronize(self.device)

    def output_ptr(self, slot):
        return lib().tmps_stage_output_ptr(self.handle, slot)

    def forward_micro(self, slot, x, y=None, labels=None, loss_out=None, stream=None):
        _check(lib().tmps_forward_micro(
            self.handle, slot, C.c_void_p(x.data_ptr()), C.c_void_p(y.data_ptr()) if y is not None else None,
            C.c_void_p(labels.data_ptr()) if labels is not None else None,
            C.c_void_p(loss_out.data_ptr()) if loss_out is not None else None, C.c_void_p(self._stream(stream))))

    def forward_micro_static(self, slot, x, y=None, labels=None, loss_out=None, stream=None):
        _check(lib().tmps_forward_micro_static(
            self.handle, slot, C.c_void_p(x.data_ptr()), C.c_void_p(y.data_ptr()) if y is not None else None,
            C.c_void_p(labels.data_ptr()) if labels is not None else None,
            C.c_void_p(loss_out.data_ptr()) if loss_out is not None else None, C.c_void_p(self._stream(stream))))

    def backward(self, slots, dy=None, dx=None, stream=None):
        arr = (C.c_int * len(slots))(*slots)
        _check(lib().tmps_backward(self.handle, arr, len(slots),
                                   C.c_void_p(dy.data_ptr()) if dy is not None else None,
                                   C.c_void_p(dx.data_ptr()) if dx is not None else None,
                                   C.c_void_p(self._stream(stream))))

    def backward_at(self, version, slots, dy=None, dx=None, stream=None):
        arr = (C.c_int * len(slots))(*slots)
        _check(lib().tmps_backward_at(self.handle, version, arr, len(slots),
                                      C.c_void_p(dy.data_ptr()) if dy is not None else None,
                                      C.c_void_p(dx.data_ptr()) if dx is not None else None,
                                      C.c_void_p(self._stream(stream))))

    def update(self, stream=None):
        _check(lib().tmps_update(self.handle, C.c_void_p(self._stream(stream))))

    def clip_gradients(self, limit, stream=None):
        """Between a backward pass and its update, on their stream: the norm of all of this stage's gradients, and the gradients clipped to it (see clip_gradients)."""
        return clip_gradients([self._flat(1, 1)], limit, stream=stream)

    def use_graphs(self, on=True):
        """Forward and backward passes replay captured HIP graphs (see tmps_stage_use_graphs)."""
        _check(lib().tmps_stage_use_graphs(self.handle, 1 if on else 0))

    def device_bytes(self):
        """Bytes of the stage's device regions: parameters (masters + working copy), optimizer state and gradients,
        activation stash, scratch, kept weight versions."""
        names = ("params", "state", "stash", "scratch")
        out = {n: int(r.numel()) for n, r in zip(names, self.regions)}
        sh = getattr(self, "shadow", None)
        out["kept_versions"] = int(sh.numel()) if sh is not None else 0
        return out


class Pipeline:
    """K stages of a workloads.Config on K streams of one GPU, run in nF1B order by tmps_schedule_run."""

    def __init__(self, cfg, params, device="cuda:0", extra_groups=0, one_stream=False, vertical_sync=False,
                 baseline_1f1b=False, batch=None, graphs=False):
        """graphs: every stage replays captured HIP graphs of its passes (for configurations of many short kernels);
        the first stage then copies its input into its stash instead of borrowing the caller's array, whose
        addresses never repeat.
        vertical_sync: forward passes read the weight version they are tagged with (the paper's vertical weight
        stashing; every stage keeps the older versions the schedule needs) instead of the live weights.
        baseline_1f1b: the comparison system instead of TiMePReSt: batches of `batch` samples (default: the
        configuration's micro-batch size), each with its own forward and backward pass, in 1F1B order, backward passes
        on the weights of their forward passes (every stage keeps the K - s - 1 older versions that takes)."""
        import torch
        self.torch = torch
        self.cfg = cfg
        self.vertical_sync = bool(vertical_sync)
        self.baseline_1f1b = bool(baseline_1f1b)
        self.device = torch.device(device)
        K, N = cfg.K, cfg.N
        self.batch = int(batch) if batch else cfg.micro
        self.stages = []
        for s in range(K):
            if self.baseline_1f1b:
                st = Stage(cfg.stages[s], cfg.dtype, self.batch, 1, K - s + extra_groups, cfg.lr, cfg.momentum,
                           borrow_input=True, device=device)
                st.set_params(params[s])
                st.set_shadow(K - s - 1)
                self.stages.append(st)
                continue
            groups = schedule_stash_groups(K, N, s) + extra_groups
            st = Stage(cfg.stages[s], cfg.dtype, cfg.micro, N, groups * N, cfg.lr, cfg.momentum,
                       borrow_input=not (graphs and s == 0), device=device)
            st.set_params(params[s])
            if graphs:
                st.use_graphs(True)
            if self.vertical_sync:
                st.set_shadow(schedule_shadow_versions(K, N, s))
            self.stages.append(st)
        # K streams created back to back by the library, so that they land on distinct hardware queues (streams from
        # torch's pool may share one, and then two workers run one after the other); wrapped for torch.
        # one_stream: every worker issues on the same stream, so kernels never overlap (for per-kernel timing)
        n = 1 if one_stream else K
        self._raw_streams = (C.c_void_p * n)()
        with torch.cuda.device(self.device):
            _check(lib().tmps_streams_create(self._raw_streams, n))
        ext = [torch.cuda.ExternalStream(int(self._raw_streams[i]), device=self.device) for i in range(n)]
        self.streams = [ext[0] if one_stream else ext[s] for s in range(K)]
        self.act_dtype = self.stages[0].act_dtype

    def __del__(self):
        raw = getattr(self, "_raw_streams", None)
        if raw is not None and _lib is not None:
            try:
                self.torch.cuda.synchronize(self.device)
                _lib.tmps_streams_destroy(raw, len(raw))
            except Exception:
                pass
            self._raw_streams = None

    def upload(self, batches):
        """Concatenate mini-batches and place them in HBM (inputs in the activation dtype, labels int32)."""
        torch = self.torch
        x = self.stages[0].prepare_input(np.concatenate([b[0] for b in batches], axis=0))
        y = torch.from_numpy(np.concatenate([b[1] for b in batches], axis=0).astype(np.int32))
        return x.contiguous(), y.to(self.device).contiguous()

    def run_device(self, x_dev, y_dev, n_minibatches, losses_dev, want_log=True, one_stream=False):
        """Launch on resident inputs.  Returns the version log (n_tasks x 7 int32) or None.
        one_stream: this run issues every worker on the first stream (kernels never share the device)."""
        K, N = self.cfg.K, self.cfg.N
        handles = (C.c_void_p * K)(*[st.handle for st in self.stages])
        streams = (C.c_void_p * K)(*[(self.streams[0] if one_stream else s).cuda_stream for s in self.streams])
        log = None
        logp = None
        if want_log:
            if self.baseline_1f1b:
                n_tasks = _check(lib().tmps_schedule_plan_1f1b(K, n_minibatches, None, 0))
            else:
                n_tasks = _check(lib().tmps_schedule_plan(K, N, n_minibatches, None, 0))
            log = (C.c_int32 * (7 * n_tasks))()
            logp = log
        if self.baseline_1f1b:   # n_minibatches counts batches here
            _check(lib().tmps_schedule_run_1f1b(handles, K, n_minibatches, C.c_void_p(x_dev.data_ptr()),
                                                C.c_void_p(y_dev.data_ptr()), streams, C.c_void_p(losses_dev.data_ptr()), logp))
        else:
            run = lib().tmps_schedule_run_vsync if self.vertical_sync else lib().tmps_schedule_run
            _check(run(handles, K, N, n_minibatches, C.c_void_p(x_dev.data_ptr()), C.c_void_p(y_dev.data_ptr()), streams,
                       C.c_void_p(losses_dev.data_ptr()), logp))
        if log is None:
            return None
        return np.frombuffer(log, dtype=np.int32).reshape(-1, 7).copy()

    def run(self, batches):
        torch = self.torch
        x, y = self.upload(batches)
        losses = torch.zeros(len(batches), dtype=torch.float32, device=self.device)
        torch.cuda.synchronize(self.device)
        log = self.run_device(x, y, len(batches), losses)
        torch.cuda.synchronize(self.device)
        return losses.cpu().numpy().tolist(), log

    def get_params(self, s):
        return self.stages[s].get_params()

    def save_checkpoint(self, directory, epoch):
        """Every stage writes its own file for `epoch` (call between runs: the pipeline is drained)."""
        return [st.save_checkpoint(directory, s, epoch) for s, st in enumerate(self.stages)]

    def resume(self, directory):
        """Load the latest epoch whose checkpoints of ALL stages are intact; returns that epoch, or None."""
        from . import checkpoint
        epoch = checkpoint.last_complete_epoch(directory, self.cfg.K)
        if epoch is None:
            return None
        for s, st in enumerate(self.stages):
            st.load_checkpoint(directory, s, epoch)
        return epoch
