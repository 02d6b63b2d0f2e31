"""The operators of a training block beside the allocators (include/vms_ops.h), for PyTorch tensors:

    dropout(x, p, seed, call, residual)     a mask that is made again wherever it is needed, and stored nowhere
    layer_norm(x, weight, bias, ...)        with the residual sum and its dropout on the way in
    low_rank_add(y, x, a, b, ...)           low-rank adapters of many requests beside a shared projection

All take float32, float16 and bfloat16 (one type for a call) on the GPU, keep their sums in 32 bits, run on the current
stream of their tensors' device and have gradients where autograd asks for them (of first order).  Outputs are new
tensors.  What is kept for the backward pass is named with each operator; a forward pass that is made again, as
recomputation does, gives the same bits.  Gradients are summed in a fixed order.

The kernels of libvmsreplay.so do all the work: wrong arguments raise ValueError or VmsError, and there is no other
path for tensors that are not on a GPU.

Tensors may have any strides.  Rows (the last dimension) that are not consecutive in memory, or leading dimensions that
are not evenly spaced, are copied first.  A call can be captured into a graph; what it allocates then belongs to the
graph.  To replay one with another mask each time, pass `seed` as a tensor and change it between the replays.
"""
import ctypes

import torch

from . import binding
from .binding import VMS_OK, VmsError

VMS_F32, VMS_F16, VMS_BF16 = 0, 1, 2
MAX_RANK = 128
_DTYPES = {torch.float32: VMS_F32, torch.float16: VMS_F16, torch.bfloat16: VMS_BF16}
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


def _call(name, args, device):
    """One call of the library on the current stream of `device`."""
    f = getattr(_lib or lib(), name)
    if device.index == torch.cuda.current_device():
        rc = f(ctypes.addressof(args), torch._C._cuda_getCurrentRawStream(device.index))
    else:
        with torch.cuda.device(device):
            rc = f(ctypes.addressof(args), torch._C._cuda_getCurrentRawStream(device.index))
    if rc != VMS_OK:
        raise VmsError(rc, name)


def _same(x, **others):
    """Every other tensor has x's type and device."""
    if x.dtype not in _DTYPES:
        raise ValueError("float32, float16 or bfloat16 tensors, got %s" % x.dtype)
    if not x.is_cuda:
        raise ValueError("tensors on a GPU, got one on %s" % x.device)
    for name, t in others.items():
        if t is not None and (t.dtype != x.dtype or t.device != x.device):
            raise ValueError("%s is %s on %s, the input %s on %s" % (name, t.dtype, t.device, x.dtype, x.device))


def _matrix(t):
    """(tensor, row stride) of t as rows of its last dimension; a copy where its strides do not allow that."""
    n = t.dim()
    if n == 2:
        if t.stride(1) == 1 or t.size(1) == 1:
            return t, t.stride(0)
    elif n == 1:
        if t.stride(0) == 1 or t.size(0) == 1:
            return t, t.size(0)
    elif t.is_contiguous():
        return t, t.size(-1)
    elif t.stride(-1) == 1 or t.size(-1) == 1:
        sizes = [(t.size(i), t.stride(i)) for i in range(n - 1) if t.size(i) != 1]
        if not sizes:
            return t, t.size(-1)
        if all(a[1] == b[0] * b[1] for a, b in zip(sizes, sizes[1:])):
            return t, sizes[-1][1]
    t = t.contiguous()
    return t, t.size(-1)


def _rows(t):
    cols = t.size(-1)
    return (t.numel() // cols if cols else 0), cols


def _ptr(t):
    return None if t is None else t.data_ptr()


def _mask(x, p, seed, call):
    if not 0.0 <= p <= 1.0:
        raise ValueError("p is a share from 0 to 1, got %r" % (p,))
    if not 0 <= call < 1 << 64:
        raise ValueError("call is a number of 64 bits, got %r" % (call,))
    if isinstance(seed, torch.Tensor):
        if seed.dtype != torch.int64 or seed.numel() != 1 or seed.device != x.device:
            raise ValueError("a seed tensor is one int64 on the input's device")
        return vms_dropout_mask(p, 0, seed.data_ptr(), call)
    if not 0 <= seed < 1 << 64:
        raise ValueError("seed is a number of 64 bits or a tensor, got %r" % (seed,))
    return vms_dropout_mask(p, seed, None, call)


def _wanted(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# ---- dropout ---------------------------------------------------------------------------------------------------------

def _dropout(x, residual, mask):
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rows, cols = _rows(x)
    m, ldx = _matrix(x)
    r, ldr = (None, 0) if residual is None else _matrix(residual)
    _call("vms_dropout", vms_dropout_args(ctypes.sizeof(vms_dropout_args), _DTYPES[x.dtype], rows, cols, m.data_ptr(), _ptr(r),
                                          y.data_ptr(), ldx, ldr, cols, mask), x.device)
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, call):
        if isinstance(seed, torch.Tensor):
            ctx.save_for_backward(seed)         # so that a seed changed before the backward pass is noticed
            ctx.rest = (p, None, call)
        else:
            ctx.rest = (p, seed, call)
        return _dropout(x, residual, _mask(x, p, seed, call))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        p, seed, call = ctx.rest
        if seed is None:
            seed, = ctx.saved_tensors
        dx = _dropout(dy, None, _mask(dy, p, seed, call)) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


def dropout(x, p, seed, call=0, residual=None):
    """residual + dropout(x), or dropout(x): a share p of the elements becomes 0, the others are divided by 1 - p.

    Which ones depends on their row (all dimensions but the last, counted through) and column, on `seed` and on `call`
    alone: 64-bit numbers of which a program gives every dropout of a step a `call` of its own and every step another
    seed.  `seed` may be an int64 tensor of one element on the same device, read when the kernel runs; it must not
    change before the backward pass.  p is taken in steps of 2^-16.  Nothing is kept for the backward pass but `seed`."""
    _same(x, residual=residual)
    if x.dim() == 0:
        raise ValueError("x has no dimension")
    if residual is not None and residual.shape != x.shape:
        raise ValueError("residual has shape %s, x %s" % (tuple(residual.shape), tuple(x.shape)))
    mask = _mask(x, p, seed, call)
    if _wanted(x, residual):
        return _Dropout.apply(x, residual, p, seed, call)
    return _dropout(x, residual, mask)


# ---- layer norm ------------------------------------------------------------------------------------------------------

def _layer_norm(x, weight, bias, eps, residual, mask, backward):
    """-> y, s (None without a residual), statistics (None without a backward pass)"""
    rows, cols = _rows(x)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    s = None if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device) if backward else None
    m, ldx = _matrix(x)
    r, ldr = (None, 0) if residual is None else _matrix(residual)
    w = None if weight is None else weight.contiguous()
    b = None if bias is None else bias.contiguous()
    _call("vms_layernorm", vms_layernorm_args(ctypes.sizeof(vms_layernorm_args), _DTYPES[x.dtype], rows, cols, m.data_ptr(), _ptr(r),
                                              _ptr(w), _ptr(b), y.data_ptr(), _ptr(s), _ptr(stats), ldx, ldr, cols, cols, eps, mask),
          x.device)
    return y, s, stats


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, eps, p, seed, call):
        y, s, stats = _layer_norm(x, weight, bias, eps, residual, _mask(x, p, seed, call), True)
        ctx.save_for_backward(x if s is None else s, stats, weight, seed if isinstance(seed, torch.Tensor) else None)
        ctx.rest = (p, seed if not isinstance(seed, torch.Tensor) else None, call)
        ctx.set_materialize_grads(False)
        return (y, s) if s is not None else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, ds=None):
        s, stats, weight, held = ctx.saved_tensors
        p, seed, call = ctx.rest
        rows, cols = _rows(s)
        new = lambda: torch.empty(s.shape, dtype=s.dtype, device=s.device)
        if dy is None:
            if ds is None:
                return (None,) * 8
            dy = torch.zeros_like(s)
        need_x, need_w, need_b, need_res = ctx.needs_input_grad[:4]
        dres = new()
        dropped = p > 0.0
        dx = new() if dropped and need_x else None
        dweight = torch.empty(cols, dtype=s.dtype, device=s.device) if need_w else None
        dbias = torch.empty(cols, dtype=s.dtype, device=s.device) if need_b else None
        m, lddy = _matrix(dy)
        e, ldds = (None, 0) if ds is None else _matrix(ds)
        k, lds = _matrix(s)
        w = None if weight is None else weight.contiguous()
        mask = _mask(s, p, seed if held is None else held, call)
        a = vms_layernorm_backward_args(ctypes.sizeof(vms_layernorm_backward_args), _DTYPES[s.dtype], rows, cols, m.data_ptr(), _ptr(e),
                                        k.data_ptr(), _ptr(w), stats.data_ptr(), dres.data_ptr(), _ptr(dx), _ptr(dweight),
                                        _ptr(dbias), lddy, ldds, lds, cols, cols, mask, None, 0)
        ws = None
        if need_w or need_b:
            a.workspace_bytes = lib().vms_layernorm_backward_workspace_bytes(ctypes.addressof(a))
            ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=s.device)
            a.d_workspace = ws.data_ptr()
        _call("vms_layernorm_backward", a, s.device)
        return ((dx if dropped else dres) if need_x else None), dweight, dbias, (dres if need_res else None), None, None, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, residual=None, p=0.0, seed=0, call=0):
    """y = (x - mean) / sqrt(variance + eps) * weight + bias over the last dimension.

    With `residual`, s = residual + dropout(x) takes x's place, and (y, s) is returned: s is the sum that the next
    residual branch goes on from.  `p`, `seed` and `call` are as in dropout().  Mean and variance are those of s before
    it is rounded.  Kept for the backward pass: s (or x), two floats for each row, `weight`."""
    _same(x, weight=weight, bias=bias, residual=residual)
    if x.dim() == 0 or x.size(-1) == 0:
        raise ValueError("x has no columns")
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None and t.shape != x.shape[-1:]:
            raise ValueError("%s has shape %s, rows have %d columns" % (name, tuple(t.shape), x.size(-1)))
    if residual is not None and residual.shape != x.shape:
        raise ValueError("residual has shape %s, x %s" % (tuple(residual.shape), tuple(x.shape)))
    if residual is None and p != 0.0:
        raise ValueError("dropout is applied on the way to the residual sum: p needs a residual")
    if not eps >= 0.0:
        raise ValueError("eps is not negative, got %r" % (eps,))
    mask = _mask(x, p, seed, call)
    if _wanted(x, weight, bias, residual):
        return _LayerNorm.apply(x, weight, bias, residual, eps, p, seed, call)
    y, s, _ = _layer_norm(x, weight, bias, eps, residual, mask, False)
    return y if s is None else (y, s)


# ---- low-rank adapters -----------------------------------------------------------------------------------------------

def _low_rank_args(x, ldx, rows, a, b, scale, starts, which):
    n, rank = (1, a.size(0)) if a.dim() == 2 else (a.size(0), a.size(1))
    scales = scale if isinstance(scale, torch.Tensor) else None
    return vms_lowrank_args(ctypes.sizeof(vms_lowrank_args), _DTYPES[x.dtype], rows, a.size(-1), b.size(-2), rank, n,
                            0 if starts is None else starts.numel() - 1, 0.0 if scales is not None else scale, _ptr(scales),
                            x.data_ptr(), None, a.data_ptr(), b.data_ptr(), _ptr(starts), _ptr(which), None, ldx, 0, 0, None, 0)


def _low_rank(y, x, a, b, scale, starts, which, inplace):
    """-> y + ..., scale * x a^T"""
    m, ldx = _matrix(x)
    base, ldy = _matrix(y)
    rows = _rows(x)[0]
    f = _low_rank_args(m, ldx, rows, a, b, scale, starts, which)
    if inplace:
        if base is not y:
            raise ValueError("y's strides do not allow the sum in place")
        out, f.ldo = y, ldy
    else:
        out, f.ldo = torch.empty(y.shape, dtype=y.dtype, device=y.device), y.size(-1)
    f.hidden_bytes = (_lib or lib()).vms_lowrank_hidden_bytes(ctypes.addressof(f))
    hidden = torch.empty(f.hidden_bytes, dtype=torch.uint8, device=x.device)
    f.d_hidden, f.d_y, f.d_out, f.ldy = hidden.data_ptr(), base.data_ptr(), out.data_ptr(), ldy
    _call("vms_lowrank", f, x.device)
    return out, hidden


class _LowRankAdd(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, x, a, b, scale, starts, which, inplace):
        out, hidden = _low_rank(y, x, a, b, scale, starts, which, inplace)
        if inplace:
            ctx.mark_dirty(y)
        tensor = isinstance(scale, torch.Tensor)
        ctx.save_for_backward(x, a, b, hidden, starts, which, scale if tensor else None)
        ctx.scale = None if tensor else scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        x, a, b, hidden, starts, which, scales = ctx.saved_tensors
        need_y, need_x, need_a, need_b = ctx.needs_input_grad[:4]
        if not (need_x or need_a or need_b):
            return dout, None, None, None, None, None, None, None
        m, ldx = _matrix(x)
        d, ldd = _matrix(dout)
        f = _low_rank_args(m, ldx, _rows(x)[0], a, b, ctx.scale if scales is None else scales, starts, which)
        f.d_hidden, f.hidden_bytes = hidden.data_ptr(), hidden.numel()
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
        da = torch.empty_like(a) if need_a else None
        db = torch.empty_like(b) if need_b else None
        g = vms_lowrank_backward_args(ctypes.sizeof(vms_lowrank_backward_args), 0, f, d.data_ptr(), _ptr(dx), _ptr(da), _ptr(db), ldd,
                                      x.size(-1), None, 0)
        g.workspace_bytes = lib().vms_lowrank_backward_workspace_bytes(ctypes.addressof(g))
        ws = torch.empty(g.workspace_bytes, dtype=torch.uint8, device=x.device)
        g.d_workspace = ws.data_ptr()
        _call("vms_lowrank_backward", g, x.device)
        return dout if need_y else None, dx, da, db, None, None, None, None


def low_rank_add(y, x, a, b, scale=1.0, starts=None, which=None, inplace=False):
    """y + scale * (x a^T) b^T: low-rank adapters beside a shared projection y of x.

    One adapter for all rows: a [rank, in], b [out, rank].  Many requests at once: a [adapters, rank, in], b [adapters,
    out, rank], and the rows of x and y packed by request: request i has rows starts[i] to starts[i + 1] - 1 and adapter
    which[i] (none if that is negative), with `starts` and `which` int32 on the device.  `starts` does not decrease; rows
    before starts[0] and from starts[-1] on belong to no request, and their sum is y.  `scale` is a number or a float32
    tensor with one for each adapter.  Ranks up to 128.

    `inplace` makes the sum in y itself and leaves rows of no request untouched.  Gradients: of y, x, a and b; an
    adapter's are summed over all its requests.  Kept for the backward pass: x, a, b, and scale * x a^T."""
    _same(x, y=y, a=a, b=b)
    if x.dim() == 0 or x.shape[:-1] != y.shape[:-1]:
        raise ValueError("x has shape %s, y %s" % (tuple(x.shape), tuple(y.shape)))
    if a.dim() != b.dim() or a.dim() not in (2, 3):
        raise ValueError("a is [rank, in] and b [out, rank], or both with the adapters in front")
    if a.shape[:-2] != b.shape[:-2] or a.size(-2) != b.size(-1) or a.size(-1) != x.size(-1) or b.size(-2) != y.size(-1):
        raise ValueError("a %s and b %s do not lead from %d to %d features" % (tuple(a.shape), tuple(b.shape), x.size(-1), y.size(-1)))
    if not 1 <= a.size(-2) <= MAX_RANK:
        raise ValueError("ranks from 1 to %d, got %d" % (MAX_RANK, a.size(-2)))
    if (starts is None) != (which is None):
        raise ValueError("starts and which come together")
    if starts is None and a.dim() == 3 and a.size(0) != 1:
        raise ValueError("several adapters need starts and which")
    if starts is not None:
        for name, t in (("starts", starts), ("which", which)):
            if t.dtype != torch.int32 or t.device != x.device or t.dim() != 1 or not t.is_contiguous():
                raise ValueError("%s is a contiguous int32 vector on the input's device" % name)
        if starts.numel() != which.numel() + 1:
            raise ValueError("%d requests have %d starts, not %d" % (which.numel(), which.numel() + 1, starts.numel()))
    if isinstance(scale, torch.Tensor):
        n = 1 if a.dim() == 2 else a.size(0)
        if scale.dtype != torch.float32 or scale.device != x.device or scale.shape != (n,) or not scale.is_contiguous():
            raise ValueError("a scale tensor is a contiguous float32 vector with one number for each adapter")
        if scale.requires_grad:
            raise ValueError("scales have no gradient")
    a, b = a.contiguous(), b.contiguous()
    if _wanted(y, x, a, b):
        return _LowRankAdd.apply(y, x, a, b, scale, starts, which, inplace)
    return _low_rank(y, x, a, b, scale, starts, which, inplace)[0]
