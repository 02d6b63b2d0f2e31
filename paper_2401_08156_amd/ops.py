"""The operators of a training block beside the allocators (include/vms_ops.h), for PyTorch tensors:

    dropout(x, p, seed, call, residual)     a mask that is made again wherever it is needed, and stored nowhere
    layer_norm(x, weight, bias, ...)        with the residual sum and its dropout on the way in
    low_rank_add(y, x, a, b, ...)           low-rank adapters of many requests beside a shared projection

All take float32, float16 and bfloat16 (one type for a call) on the GPU, keep their sums in 32 bits, run on the current
stream of their tensors' device and have gradients where autograd asks for them (of first order).  Outputs are new
tensors.  What is kept for the backward pass is named with each operator; a forward pass that is made again, as
recomputation does, gives the same bits.  Gradients are summed in a fixed order.

The kernels of libvmsreplay.so do all the work, called from the autograd nodes of _vms_torch.so (csrc/vms_torch_ops.cpp):
wrong arguments raise ValueError or VmsError, and there is no other path for tensors that are not on a GPU.  PyTorch does not
see what they compute: traces (torch.jit.trace, make_fx) and forward-mode gradients are refused.  The structures
below are those of the C entry points, for programs that call them with pointers of their own.

Tensors may have any strides.  Rows (the last dimension) that are not consecutive in memory, leading dimensions that are not
evenly spaced, and rows 2^31 elements apart (2^23 for adapters) are copied first.  A call can be captured into a graph; what it allocates then belongs to the
graph.  To replay one with another mask each time, pass `seed` as a tensor and change it between the replays.  As with every
operator, a backward pass is captured only while no eager graph of the same leaves is alive.
"""
import ctypes
import importlib.util
import os

from . import binding
from . import build as _build
from .binding import VmsError

VMS_F32, VMS_F16, VMS_BF16 = 0, 1, 2
MAX_RANK = 128
_u32, _u64, _vp, _f32, _f64 = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_float, ctypes.c_double


class vms_dropout_mask(ctypes.Structure):
    _fields_ = [("p", _f64), ("seed", _u64), ("d_seed", _vp), ("call", _u64)]


class vms_dropout_args(ctypes.Structure):
    _fields_ = [("struct_size", _u32), ("dtype", _u32), ("rows", _u64), ("cols", _u64),
                ("d_x", _vp), ("d_residual", _vp), ("d_y", _vp),
                ("ldx", _u64), ("ldr", _u64), ("ldy", _u64), ("mask", vms_dropout_mask)]


class vms_layernorm_args(ctypes.Structure):
    _fields_ = [("struct_size", _u32), ("dtype", _u32), ("rows", _u64), ("cols", _u64),
                ("d_x", _vp), ("d_residual", _vp), ("d_weight", _vp), ("d_bias", _vp), ("d_y", _vp), ("d_s", _vp),
                ("d_stats", _vp), ("ldx", _u64), ("ldr", _u64), ("ldy", _u64), ("lds", _u64), ("eps", _f64),
                ("mask", vms_dropout_mask)]


class vms_layernorm_backward_args(ctypes.Structure):
    _fields_ = [("struct_size", _u32), ("dtype", _u32), ("rows", _u64), ("cols", _u64),
                ("d_dy", _vp), ("d_ds", _vp), ("d_s", _vp), ("d_weight", _vp), ("d_stats", _vp),
                ("d_dres", _vp), ("d_dx", _vp), ("d_dweight", _vp), ("d_dbias", _vp),
                ("lddy", _u64), ("ldds", _u64), ("lds", _u64), ("lddres", _u64), ("lddx", _u64),
                ("mask", vms_dropout_mask), ("d_workspace", _vp), ("workspace_bytes", _u64)]


class vms_lowrank_args(ctypes.Structure):
    _fields_ = [("struct_size", _u32), ("dtype", _u32), ("rows", _u64), ("in_", _u64), ("out", _u64),
                ("rank", _u32), ("n_adapters", _u32), ("n_requests", _u32), ("scale", _f32), ("d_scales", _vp),
                ("d_x", _vp), ("d_y", _vp), ("d_a", _vp), ("d_b", _vp), ("d_starts", _vp), ("d_which", _vp),
                ("d_out", _vp), ("ldx", _u64), ("ldy", _u64), ("ldo", _u64), ("d_hidden", _vp), ("hidden_bytes", _u64)]


class vms_lowrank_backward_args(ctypes.Structure):
    _fields_ = [("struct_size", _u32), ("reserved0", _u32), ("f", vms_lowrank_args), ("d_dout", _vp),
                ("d_dx", _vp), ("d_da", _vp), ("d_db", _vp), ("lddout", _u64), ("lddx", _u64),
                ("d_workspace", _vp), ("workspace_bytes", _u64)]


EXPORTS = ["vms_dropout", "vms_layernorm", "vms_layernorm_backward", "vms_layernorm_backward_workspace_bytes",
           "vms_lowrank", "vms_lowrank_hidden_bytes", "vms_lowrank_backward", "vms_lowrank_backward_workspace_bytes"]

_lib = None


def lib():
    """libvmsreplay.so with the signatures of include/vms_ops.h."""
    global _lib
    if _lib is None:
        L = binding.lib()
        for name in EXPORTS:
            f = getattr(L, name)
            if name.endswith("_bytes"):
                f.restype, f.argtypes = ctypes.c_size_t, [_vp]
            else:
                f.restype, f.argtypes = ctypes.c_int, [_vp, _vp]
        _lib = L
    return _lib


_nodes = None


def nodes():
    """The module of autograd nodes (built in-tree; built now only if it is missing)."""
    global _nodes
    if _nodes is None:
        if not os.path.exists(_build.EXT):
            _build.build()
        binding.lib()
        spec = importlib.util.spec_from_file_location("_vms_torch", _build.EXT)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.raise_as(VmsError)
        _nodes = module
    return _nodes


def dropout(x, p, seed, call=0, residual=None):
    """residual + dropout(x), or dropout(x): a share p of the elements becomes 0, the others are divided by 1 - p.

    Which ones depends on their row (all dimensions but the last, counted through) and column, on `seed` and on `call`
    alone: 64-bit numbers of which a program gives every dropout of a step a `call` of its own and every step another
    seed.  `seed` may be an int64 tensor of one element on the same device, whose 64 bits are read when the kernel runs; it must not
    change before the backward pass.  p is taken in steps of 2^-16.  Nothing is kept for the backward pass but `seed`."""
    return (_nodes or nodes()).dropout(x, p, seed, call, residual)


def layer_norm(x, weight=None, bias=None, eps=1e-5, residual=None, p=0.0, seed=0, call=0):
    """y = (x - mean) / sqrt(variance + eps) * weight + bias over the last dimension.

    With `residual`, s = residual + dropout(x) takes x's place, and (y, s) is returned: s is the sum that the next
    residual branch goes on from.  `p`, `seed` and `call` are as in dropout().  y goes by s before it is rounded, the
    gradients by s as it is returned.  Kept for the backward pass: s (or x), two floats for each row, `weight`."""
    return (_nodes or nodes()).layer_norm(x, weight, bias, eps, residual, p, seed, call)


def low_rank_add(y, x, a, b, scale=1.0, starts=None, which=None, inplace=False):
    """y + scale * (x a^T) b^T: low-rank adapters beside a shared projection y of x.

    One adapter for all rows: a [rank, in], b [out, rank].  Many requests at once: a [adapters, rank, in], b [adapters,
    out, rank], and the rows of x and y packed by request: request i has rows starts[i] to starts[i + 1] - 1 and adapter
    which[i] (none if that is negative), with `starts` and `which` int32 on the device.  `starts` does not decrease; rows
    before starts[0] and from starts[-1] on belong to no request, and their sum is y.  `scale` is a number or a float32
    tensor with one for each adapter.  Ranks up to 128, adapters and requests up to 65535.

    `inplace` makes the sum in y itself and leaves rows of no request untouched; what lies in y's memory of the other tensors
    (x may be y) is copied first.  Gradients: of y, x, a and b; an
    adapter's are summed over all its requests.  Kept for the backward pass: x, a, b, and scale * x a^T."""
    return (_nodes or nodes()).low_rank_add(y, x, a, b, scale, starts, which, inplace)
