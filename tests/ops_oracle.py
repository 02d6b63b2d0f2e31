"""The operators of paper_2401_08156_amd/ops.py in 64 bits on the CPU, written from their definitions, and how far a
kernel that keeps its sums in 32 bits may be from them.  Shares no code with the package.

Rounding to a type is off by at most u = finfo.eps / 2 of the value (below the smallest normal number, half the
smallest subnormal one); every operation in 32 bits by 2^-24, and the matrix instructions, whose inner sums are not
specified to be rounded to nearest, by 2^-23 for each step of 4 to 32 products.
"""
import numpy as np
import torch

E32, EMMA = 2.0 ** -24, 2.0 ** -23
M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
# roundings that a value passes through in a sum over a row: elements of a lane, lanes, wavefronts
DEPTH = 64


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """half the smallest subnormal number"""
    f = torch.finfo(dtype)
    return f.tiny * f.eps / 2


def philox(counter, key):
    """Philox-4x32 with ten rounds on one counter of four words."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(10):
        p0, p1 = M0 * c[0], M1 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return c


def numbers(rows, cols, seed, call):
    """the 16-bit number of every element, [rows, cols]"""
    u64 = np.uint64
    group = np.arange((cols + 7) // 8, dtype=u64)[None, :]
    shape = (rows, group.shape[1])
    c = [np.broadcast_to(group, shape), np.broadcast_to(np.arange(rows, dtype=u64)[:, None], shape),
         np.full(shape, call & 0xFFFFFFFF, u64), np.full(shape, call >> 32, u64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    low = u64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * u64(M0), c[2] * u64(M1)
        c = [(p1 >> u64(32)) ^ c[1] ^ u64(k[0]), p1 & low, (p0 >> u64(32)) ^ c[3] ^ u64(k[1]), p0 & low]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    halves = [h for w in c for h in (w & u64(0xFFFF), w >> u64(16))]
    return np.stack(halves, axis=-1).reshape(rows, -1)[:, :cols].astype(np.int64)


def mask(shape, p, seed, call):
    """(kept, factor): truth values in the tensor's shape, and what is kept is multiplied by"""
    limit = int(np.floor(p * 65536 + 0.5))
    rows = int(np.prod(shape[:-1], dtype=np.int64))
    kept = torch.from_numpy(numbers(rows, shape[-1], seed, call) >= limit).reshape(shape)
    return kept, (65536.0 / (65536 - limit) if limit < 65536 else 0.0)


def drop(v, kept, factor):
    return torch.where(kept, v * factor, torch.zeros((), dtype=v.dtype))


def dropout(x, p, seed, call, residual=None):
    kept, factor = mask(x.shape, p, seed, call)
    y = drop(x, kept, factor)
    return y if residual is None else residual + y


def norm(x, weight, bias, eps, residual=None, p=0.0, seed=0, call=0):
    """-> y, s, and what the backward pass goes on from"""
    s = x if residual is None else dropout(x, p, seed, call, residual)
    mean = s.mean(-1, keepdim=True)
    q = 1.0 / torch.sqrt(((s - mean) ** 2).mean(-1, keepdim=True) + eps)
    h = (s - mean) * q
    y = h if weight is None else h * weight
    return (y if bias is None else y + bias), s, (h, q)


def norm_backward(dy, ds, saved, weight, x_shape, p=0.0, seed=0, call=0):
    """-> dx, dresidual, dweight, dbias"""
    h, q = saved
    g = dy if weight is None else dy * weight
    dres = q * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    if ds is not None:
        dres = dres + ds
    kept, factor = mask(x_shape, p, seed, call)
    rows = tuple(range(dy.dim() - 1))
    return drop(dres, kept, factor), dres, (dy * h).sum(rows), dy.sum(rows)


def norm_bounds(dtype, x, weight, bias, residual, factor, y, s, saved):
    """How far y and s may be off.  s: two roundings in 32 bits and one to the type.  The mean: DEPTH roundings of values
    up to `top`; s - mean: those and its own.  The variance's relative error: DEPTH, and twice that of s - mean over its
    size; q has half of it."""
    u = unit(dtype)
    h, q = saved
    size = x.abs() * factor + (0.0 if residual is None else residual.abs())
    top = size.amax(-1, keepdim=True)
    w = torch.ones_like(h) if weight is None else weight.abs().expand_as(h)
    b = torch.zeros_like(h) if bias is None else bias.abs().expand_as(h)
    e_h = E32 * (DEPTH * top * q + h.abs() * (DEPTH + DEPTH * top * q))
    e_y = u * y.abs() + e_h * w + 4 * E32 * ((h * w).abs() + b) + tiny(dtype)
    e_s = u * s.abs() + 2 * E32 * size + tiny(dtype)
    return e_y, e_s, e_h


def norm_backward_bounds(dtype, dy, ds, saved, weight, grads, e_h, factor, depth=256):
    """How far the gradients at a given s may be off: e_h is the bound of its normalised values."""
    u = unit(dtype)
    h, q = saved
    dx, dres, dw, db = grads
    g = dy.abs() if weight is None else (dy * weight).abs()
    e = e_h
    c1, c2 = g.mean(-1, keepdim=True), (g * h.abs()).mean(-1, keepdim=True)
    e_c1 = (DEPTH + 1) * E32 * c1
    e_c2 = (g * e).mean(-1, keepdim=True) + (DEPTH + 2) * E32 * c2
    parts = q * (g + c1 + h.abs() * c2)
    e_q = E32 * (DEPTH + 4) + e_h.amax(-1, keepdim=True)      # relative error of q, which e_h holds once more
    e_core = q * (e_c1 + (h.abs() + e) * e_c2 + e * c2) + parts * (e_q + 8 * E32)
    if ds is not None:
        e_core = e_core + 2 * E32 * ds.abs()
    rows = tuple(range(dy.dim() - 1))
    return (u * dx.abs() + (e_core + 2 * E32 * dres.abs()) * factor + tiny(dtype), u * dres.abs() + e_core + tiny(dtype),
            u * dw.abs() + (dy.abs() * e).sum(rows) + depth * E32 * (dy * h).abs().sum(rows) + tiny(dtype),
            u * db.abs() + depth * E32 * dy.abs().sum(rows) + tiny(dtype))


def parts_of(rows, starts, which, adapters):
    """(first row, row behind the last, adapter) of every request that has one"""
    if starts is None:
        return [(0, rows, 0)]
    return [(lo, hi, k) for lo, hi, k in zip(starts[:-1], starts[1:], which) if 0 <= k < adapters and hi > lo]


def low_rank(dtype, y, x, a, b, scale, starts=None, which=None, dout=None):
    """-> {name: (value, how far it may be off)} of out and, with dout, dx, da, db; x, y, dout are matrices, a and b have
    the adapters in front, scale is a list with one for each.

    hidden is a sum in 32 bits over `in` products, rounded to the type where that has 16 bits; a sum over n products
    passes through at most n / 16 matrix steps and DEPTH more additions."""
    u = unit(dtype)
    u_h = 0.0 if dtype == torch.float32 else u
    zero = 0.0 if dtype == torch.float32 else tiny(dtype)
    chain = lambda n: (n / 4 + DEPTH) * EMMA
    out, e_out = y.clone(), torch.zeros_like(y)
    grads = {n: [torch.zeros_like(v), torch.zeros_like(v)] for n, v in (("dx", x), ("da", a), ("db", b))}
    for lo, hi, k in parts_of(x.size(0), starts, which, a.size(0)):
        xs, ak, bk, sc = x[lo:hi], a[k], b[k], scale[k]
        h = sc * (xs @ ak.t())
        size = abs(sc) * (xs.abs() @ ak.abs().t())
        e_h = (chain(x.size(1)) + 2 * E32) * size
        e_hr = e_h + u_h * (h.abs() + e_h) + zero
        out[lo:hi] += h @ bk.t()
        e_out[lo:hi] = e_hr @ bk.abs().t() + chain(a.size(1)) * ((h.abs() + e_hr) @ bk.abs().t()) + 2 * E32 * y[lo:hi].abs()
        if dout is None:
            continue
        d = dout[lo:hi]
        dh = sc * (d @ bk)
        e_d = (chain(b.size(1)) + 2 * E32) * (abs(sc) * (d.abs() @ bk.abs()))
        e_dr = e_d + u_h * (dh.abs() + e_d) + zero
        grads["dx"][0][lo:hi] = dh @ ak
        grads["dx"][1][lo:hi] = e_dr @ ak.abs() + chain(a.size(1)) * ((dh.abs() + e_dr) @ ak.abs())
        n = x.size(0)
        grads["da"][0][k] += dh.t() @ xs
        grads["da"][1][k] += e_dr.t() @ xs.abs() + chain(n) * ((dh.abs() + e_dr).t() @ xs.abs())
        grads["db"][0][k] += d.t() @ h
        grads["db"][1][k] += d.abs().t() @ e_hr + chain(n) * (d.abs().t() @ (h.abs() + e_hr))
    got = dict(out=(out, u * out.abs() + (1 + u) * e_out + tiny(dtype)))
    if dout is not None:
        for n, (v, e) in grads.items():
            got[n] = (v, u * v.abs() + (1 + u) * e + tiny(dtype))
    return got


def assert_within(name, got, want, bound):
    """`got` (a GPU tensor) is within `bound` of `want`, and neither has other infinities or NaN"""
    g = got.detach().cpu().double()
    assert g.shape == want.shape, (name, g.shape, want.shape)
    if not g.numel():
        return
    assert torch.equal(torch.isnan(g), torch.isnan(want)), "%s: NaN in other places" % name
    fine = torch.isfinite(want)
    assert torch.equal(g[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), "%s: infinities in other places" % name
    off = ((g - want).abs() - bound)[fine]
    if off.numel():
        assert off.max() <= 0, "%s: %d of %d outside, by %.3g at most, where %.3g is allowed" % (
            name, int((off > 0).sum()), off.numel(), float(off.max()), float(bound.expand_as(want)[fine][off.argmax()]))
