"""The operators on the GPU against the oracle in 64 bits (ops_oracle.py, where the tolerances are derived)."""
import pytest
import torch

import ops_oracle as oo
from paper_2401_08156_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
ids = lambda v: str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None
SEED, CALL = 0x9E3779B97F4A7C15, (3 << 32) + 11


def normal(shape, dtype, seed, by=1.0, around=0.0):
    """(the tensor on the GPU, the same values in 64 bits)"""
    g = torch.Generator().manual_seed(seed)
    t = (torch.randn(shape, generator=g, dtype=torch.float64) * by + around).to(dtype)
    return t.cuda(), t.double()


# ---- dropout ---------------------------------------------------------------------------------------------------------

def check_dropout(y, x, p, dtype, residual=None, seed=SEED, call=CALL):
    want = oo.dropout(x, p, seed, call, residual)
    _, factor = oo.mask(x.shape, p, seed, call)
    size = x.abs() * factor + (0.0 if residual is None else residual.abs())
    oo.assert_within("y", y, want, oo.unit(dtype) * want.abs() + 2 * oo.E32 * size + oo.tiny(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (5, 8), (1, 65), (2, 1001), (300, 64), (3, 4, 50), (17,), (4096, 9), (1, 70001)])
def test_dropout_and_its_gradients(shape, dtype):
    p = 0.3
    x, x64 = normal(shape, dtype, 1)
    r, r64 = normal(shape, dtype, 2)
    dy, dy64 = normal(shape, dtype, 3)
    x.requires_grad_(True)
    r.requires_grad_(True)
    for res, res64 in ((None, None), (r, r64)):
        y = ops.dropout(x, p, SEED, CALL, residual=res)
        assert y.dtype == dtype and y.shape == x.shape
        check_dropout(y, x64, p, dtype, res64)
        grads = torch.autograd.grad(y, [x] if res is None else [x, res], dy)
        check_dropout(grads[0], dy64, p, dtype)
        if res is not None:
            assert torch.equal(grads[1], dy)
        with torch.no_grad():
            assert torch.equal(ops.dropout(x, p, SEED, CALL, residual=res), y)


@pytest.mark.parametrize("p", [0.0, 1e-6, 2.0 ** -16, 0.5, 0.999, 1.0])
def test_dropout_shares(p):
    x, x64 = normal((37, 129), torch.float32, 4)
    check_dropout(ops.dropout(x, p, 1, 0), x64, p, torch.float32, seed=1, call=0)
    if p in (0.0, 1e-6):
        assert torch.equal(ops.dropout(x, p, 1, 0), x)
    if p == 1.0:
        assert not ops.dropout(x, p, 1, 0).any()


def test_dropout_depends_on_place_seed_and_call_alone():
    kept = lambda y: y != 0
    one = lambda dtype: torch.ones(64, 40, dtype=dtype, device="cuda")
    base = kept(ops.dropout(one(torch.float32), 0.5, SEED, CALL))
    for dtype in TYPES:
        assert torch.equal(kept(ops.dropout(one(dtype), 0.5, SEED, CALL)), base)
    wide = torch.ones(64, 100, device="cuda")[:, 3:43]
    assert torch.equal(kept(ops.dropout(wide, 0.5, SEED, CALL)), base)
    assert torch.equal(kept(ops.dropout(one(torch.float32)[:31], 0.5, SEED, CALL)), base[:31])
    for seed, call in ((SEED + 1, CALL), (SEED, CALL + 1), (SEED ^ (1 << 40), CALL), (SEED, CALL ^ (1 << 32))):
        other = kept(ops.dropout(one(torch.float32), 0.5, seed, call))
        # 2560 independent pairs, equal with a chance of 1/2: six standard deviations of the share are 0.06
        assert abs(float((other == base).double().mean()) - 0.5) < 0.06


def test_dropped_infinities_and_nan_are_gone():
    kept, _ = oo.mask((16, 33), 0.5, SEED, CALL)
    x = torch.where(kept, 1.0, float("nan")).float()
    x[0] = torch.where(kept[0], 1.0, float("inf"))
    y = ops.dropout(x.cuda(), 0.5, SEED, CALL).cpu()
    assert torch.equal(y, torch.where(kept, 2.0, 0.0))


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_dropout_strides_and_empty_tensors(dtype):
    base, base64 = normal((9, 5, 24), dtype, 5)
    for cut in (lambda t: t[:, :, 1:20], lambda t: t[:, 1:3], lambda t: t.transpose(0, 2), lambda t: t[0, 0].expand(6, 24), lambda t: t[::2]):
        check_dropout(ops.dropout(cut(base), 0.25, SEED, CALL), cut(base64), 0.25, dtype)
        check_dropout(ops.dropout(cut(base), 0.25, SEED, CALL, residual=cut(base)), cut(base64), 0.25, dtype, cut(base64))
    for shape in ((0, 8), (8, 0), (0,)):
        x = torch.zeros(shape, dtype=dtype, device="cuda", requires_grad=True)
        y = ops.dropout(x, 0.5, 1)
        y.sum().backward()
        assert y.shape == x.grad.shape == shape


def test_dropout_of_rows_far_apart():
    # the last row begins behind 2^32 elements
    far = torch.empty(4 << 31, dtype=torch.bfloat16, device="cuda")
    x, x64 = normal((4, 100), torch.bfloat16, 6)
    view = torch.as_strided(far, (4, 100), ((1 << 31) - 8, 1))
    view.copy_(x)
    check_dropout(ops.dropout(view, 0.5, SEED, CALL), x64, 0.5, torch.bfloat16)
    y = ops.layer_norm(view)
    want, s, saved = oo.norm(x64, None, None, 1e-5)
    oo.assert_within("y", y, want, oo.norm_bounds(torch.bfloat16, x64, None, None, None, 1.0, want, s, saved)[0])


def test_seed_in_device_memory_and_its_change_before_the_backward_pass():
    seed = torch.tensor([12345], dtype=torch.int64, device="cuda")
    x, x64 = normal((40, 64), torch.float32, 7)
    x.requires_grad_(True)
    check_dropout(ops.dropout(x, 0.4, seed, 2), x64, 0.4, torch.float32, seed=12345, call=2)
    seed.fill_(-7)
    y = ops.dropout(x, 0.4, seed, 2)
    check_dropout(y, x64, 0.4, torch.float32, seed=(1 << 64) - 7, call=2)
    seed.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


# ---- layer norm ------------------------------------------------------------------------------------------------------

def check_norm(shape, dtype, affine=True, bias=True, residual=True, p=0.2, use_s=True, eps=1e-5, around=0.0, cut=None, small=False):
    cut = cut or (lambda t: t)
    cols = cut(torch.empty(shape)).shape[-1]
    (x, x64), (r, r64), (dy, dy64), (ds, ds64) = [[cut(t) for t in normal(shape, dtype, s, around=around if s < 3 else 0.0)] for s in (1, 2, 3, 4)]
    w, w64 = normal((cols,), dtype, 5, 0.2, 1.0) if affine else (None, None)
    b, b64 = normal((cols,), dtype, 6, 0.2) if bias else (None, None)
    if not residual:
        r = r64 = None
    p = p if residual else 0.0
    leaves = [t.detach().requires_grad_(True) for t in (x, w, b, r) if t is not None]
    it = iter(leaves)
    x, w, b, r = [next(it) if t is not None else None for t in (x, w, b, r)]
    got = ops.layer_norm(x, w, b, eps, residual=r, p=p, seed=SEED, call=CALL)
    y, s = got if residual else (got, None)
    want, s64, saved = oo.norm(x64, w64, b64, eps, r64, p, SEED, CALL)
    _, factor = oo.mask(x64.shape, p, SEED, CALL)
    e_y, e_s, _ = oo.norm_bounds(dtype, x64, w64, b64, r64, factor, want, s64, saved)
    oo.assert_within("y", y, want, e_y)
    if residual:
        oo.assert_within("s", s, s64, e_s)
    with torch.no_grad():
        again = ops.layer_norm(x, w, b, eps, residual=r, p=p, seed=SEED, call=CALL)
        assert all(torch.equal(u, v) for u, v in zip(again if residual else (again,), (y, s)))
    outs, grads = ([y, s], [dy, ds]) if residual and use_s else ([y], [dy])
    ds64 = ds64 if residual and use_s else None
    got = dict(zip([n for n, t in (("x", x), ("w", w), ("b", b), ("r", r)) if t is not None], torch.autograd.grad(outs, leaves, grads)))
    # the gradients are those at the sum that the forward pass returned
    at = s.detach().cpu().double() if residual else x64
    here, _, saved = oo.norm(at, w64, b64, eps)
    e_h = oo.norm_bounds(dtype, at, w64, b64, None, 1.0, here, at, saved)[2]
    want = oo.norm_backward(dy64, ds64, saved, w64, x64.shape, p, SEED, CALL)
    bounds = oo.norm_backward_bounds(dtype, dy64, ds64, saved, w64, want, e_h, factor)
    for n, v, e in zip("xrwb", want, bounds):
        if n in got:
            assert got[n].dtype == dtype
            oo.assert_within("gradient of " + n, got[n], v, e)


# every kernel variant: rows of a wavefront, of 256 to 1024 lanes, and longer ones than registers hold
COLS = [1, 2, 7, 8, 63, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8191, 8200, 16384, 16385, 32768, 32776, 40001]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("cols", COLS)
def test_layer_norm_and_its_gradients(cols, dtype):
    check_norm((5, cols), dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("kw", [dict(affine=False, bias=False), dict(affine=False), dict(bias=False), dict(residual=False),
                                dict(residual=False, affine=False, bias=False), dict(p=0.0), dict(use_s=False), dict(p=1.0), dict(eps=0.5)],
                         ids=lambda kw: "-".join("%s=%s" % i for i in kw.items()))
def test_layer_norm_with_parts_left_out(kw, dtype):
    check_norm((2, 3, 200), dtype, **kw)
    check_norm((7, 4100), dtype, **kw)


@pytest.mark.parametrize("rows,cols", [(1, 4096), (1, 8), (2050, 33), (5000, 512), (1500, 2056), (700, 8192), (300, 16384), (300, 32776)])
def test_layer_norm_of_more_rows_than_workgroups(rows, cols):
    check_norm((rows, cols), torch.bfloat16)


@pytest.mark.parametrize("cols", [600, 5000, 33000])
def test_layer_norm_of_rows_far_from_zero(cols):
    # a mean of 1000 deviations: the variance is not a difference of squares
    check_norm((6, cols), torch.float32, around=1000.0, residual=False)


def test_layer_norm_strides():
    for cut in (lambda t: t[..., 3:77], lambda t: t[:, 1:3], lambda t: t.transpose(0, 1), lambda t: t[::2]):
        check_norm((6, 4, 90), torch.float16, cut=cut)


def test_layer_norm_of_equal_values_infinities_and_nan():
    x = torch.ones(4, 100, device="cuda") * 3.0
    x[1, 5] = float("inf")
    x[2, 99] = float("nan")
    y = ops.layer_norm(x, eps=1e-5)
    assert not y[0].any() and not y[3].any() and torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
    w = torch.ones(100, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(ops.layer_norm(x[::3], w), w, torch.ones(2, 100, device="cuda"))
    assert not g.any()


def test_layer_norm_without_rows():
    for dtype in TYPES:
        x = torch.zeros(0, 24, dtype=dtype, device="cuda", requires_grad=True)
        w, b = [torch.ones(24, dtype=dtype, device="cuda", requires_grad=True) for _ in range(2)]
        junk = torch.full((1 << 16,), 7.0, device="cuda")
        del junk
        y = ops.layer_norm(x, w, b)
        gx, gw, gb = torch.autograd.grad(y, (x, w, b), torch.zeros_like(y))
        assert gx.shape == (0, 24) and not gw.any() and not gb.any()


def test_layer_norm_gradients_that_nobody_asks_for():
    x, x64 = normal((33, 1000), torch.bfloat16, 1)
    w, w64 = normal((1000,), torch.bfloat16, 2, 0.1, 1.0)
    r, _ = normal((33, 1000), torch.bfloat16, 3)
    dy, _ = normal((33, 1000), torch.bfloat16, 4)
    for leaves in ([x], [w], [r], [x, r]):
        for t in (x, w, r):
            t.requires_grad_(any(t is v for v in leaves))
        y, s = ops.layer_norm(x, w, residual=r, p=0.1, seed=1)
        some = torch.autograd.grad(y, leaves, dy)
        for t in (x, w, r):
            t.requires_grad_(True)
        y, s = ops.layer_norm(x, w, residual=r, p=0.1, seed=1)
        assert all(torch.equal(u, v) for u, v in zip(some, torch.autograd.grad(y, leaves, dy)))
    for t in (x, w, r):
        t.requires_grad_(True)
    y, s = ops.layer_norm(x, w, residual=r, p=0.1, seed=1)
    gs = torch.autograd.grad(s, [x, r], dy)          # only the sum is used
    check_dropout(gs[0], dy.cpu().double(), 0.1, torch.bfloat16, seed=1, call=0)
    assert torch.equal(gs[1], dy)


# ---- low-rank adapters -----------------------------------------------------------------------------------------------

def check_low_rank(rows, k, n, rank, dtype, adapters=1, starts=None, which=None, scale=0.5, cut=None, inplace=False, step=True, flat=False):
    cut = cut or (lambda t: t)
    x, x64 = [cut(t) for t in normal((rows, k), dtype, 1)]
    y, y64 = [cut(t) for t in normal((rows, n), dtype, 2)]
    dout, dout64 = [cut(t) for t in normal((rows, n), dtype, 5)]
    k, n = x.shape[1], y.shape[1]
    a, a64 = normal((adapters, rank, k), dtype, 3, k ** -0.5)
    b, b64 = normal((adapters, n, rank), dtype, 4, rank ** -0.5)
    scales = torch.tensor(scale, dtype=torch.float32, device="cuda") if isinstance(scale, list) else scale
    s = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    w = None if starts is None else torch.tensor(which, dtype=torch.int32, device="cuda")
    if flat:
        a, b = a[0], b[0]
    want = oo.low_rank(dtype, y64, x64, a64, b64, scale if isinstance(scale, list) else [scale] * adapters, starts, which, dout64 if step else None)
    leaves = [t.detach().requires_grad_(step) for t in (x, a, b, y)]
    into = leaves[3].clone() if inplace else leaves[3]
    out = ops.low_rank_add(into, *leaves[:3], scale=scales, starts=s, which=w, inplace=inplace)
    assert out.dtype == dtype and (out is into or not inplace)
    oo.assert_within("out", out, *want["out"])
    if not step:
        return
    got = torch.autograd.grad(out, leaves, dout)
    for name, g in zip(("dx", "da", "db"), got):
        v, e = want[name]
        if flat and name != "dx":
            v, e = v[0], e[0]
        oo.assert_within(name, g, v, e)
    assert torch.equal(got[3], dout)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,k,n,rank", [(1, 1, 1, 1), (1, 64, 64, 16), (3, 33, 17, 5), (16, 256, 128, 16), (17, 100, 300, 12), (65, 513, 129, 24),
                                           (200, 1024, 512, 64), (130, 96, 1000, 100), (257, 640, 320, 128), (1000, 70, 90, 8), (4, 5000, 4100, 33)])
def test_one_adapter(rows, k, n, rank, dtype):
    check_low_rank(rows, k, n, rank, dtype, flat=True)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("starts,which", [
    ([0, 1, 2, 3, 4, 5], [2, 0, 1, -1, 2]),                     # single tokens, one of them without an adapter
    ([0, 70, 70, 75, 200], [1, 0, 0, 2]),                       # an empty request, adapters used again
    ([3, 40, 111], [2, 2]),                                     # rows before the first request and behind the last
    ([0, 0, 0], [1, 1]),                                        # nothing but rows without a request
    ([0, 300], [7]),                                            # a number that no adapter has
])
def test_many_requests(starts, which, dtype):
    rows = max(starts[-1], 5) + 9
    for rank in (4, 40):
        check_low_rank(rows, 136, 200, rank, dtype, 3, starts, which, scale=[0.5, -1.0, 2.0])


def test_requests_of_all_tile_sizes_and_more_than_a_wavefront_counts():
    g = torch.Generator().manual_seed(1)
    for most, count in ((2, 150), (60, 40), (200, 9)):
        lengths = torch.randint(0, most, (count,), generator=g)
        starts = [0] + torch.cumsum(lengths, 0).tolist()
        which = torch.randint(-1, 5, (count,), generator=g).tolist()
        check_low_rank(starts[-1] + 3, 160, 96, 16, torch.bfloat16, 5, starts, which)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rank", [8, 16, 32, 64, 128])
def test_short_requests_beside_a_longer_one(rank, dtype):
    lengths = [1, 2, 1, 0, 3, 1, 1, 9, 1, 1, 1, 2]
    starts = [2]
    for n in lengths:
        starts.append(starts[-1] + n)
    which = [0, 1, 2, 0, 0, -1, 2, 1, 1, 0, 5, 2]
    check_low_rank(starts[-1] + 1, 300, 333, rank, dtype, 3, starts, which, scale=[1.0, 0.5, -2.0], step=rank == 16)
    check_low_rank(2, 64, 1000, rank, dtype, flat=True, step=False)
    check_low_rank(starts[-1] + 1, 300, 333, rank, dtype, 3, starts, which, inplace=True, step=False)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rank", [3, 20, 50, 100, 127])
def test_few_rows_and_every_padded_rank(rank, dtype):
    check_low_rank(7, 520, 700, rank, dtype, flat=True)
    check_low_rank(60, 130, 260, rank, dtype, 2, [0, 20, 25, 57], [1, 0, 1])


def test_numbers_of_numpy_as_seeds():
    import numpy as np
    x, x64 = normal((5, 40), torch.float32, 1)
    check_dropout(ops.dropout(x, np.float64(0.5), np.int64(3), np.uint32(4)), x64, 0.5, torch.float32, seed=3, call=4)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_outputs_larger_than_the_last_cache(dtype):
    # (accesses marked as not to be kept) the oracle sees some rows; the sums over all rows are left to the other tests
    n = 4096 if dtype == torch.float32 else 8192
    rows = (300 << 20) // (3 * n * (4 if dtype == torch.float32 else 2))
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    x, r, dy, ds = [new(rows, n).requires_grad_(i < 2) for i in range(4)]
    w = new(n).requires_grad_(True)
    some = torch.tensor([0, 1, rows // 2, rows - 1])
    kept, factor = oo.mask((rows, n), 0.3, SEED, CALL)
    x64, r64, dy64, ds64 = [t.detach()[some.cuda()].cpu().double() for t in (x, r, dy, ds)]
    s64 = r64 + oo.drop(x64, kept[some], factor)
    y = ops.dropout(x, 0.3, SEED, CALL, residual=r)
    size = x64.abs() * factor + r64.abs()
    oo.assert_within("dropout", y[some.cuda()], s64, oo.unit(dtype) * s64.abs() + 2 * oo.E32 * size + oo.tiny(dtype))
    y, s = ops.layer_norm(x, w, residual=r, p=0.3, seed=SEED, call=CALL)
    w64 = w.detach().cpu().double()
    want, _, saved = oo.norm(s64, w64, None, 1e-5)
    e_y, e_s, _ = oo.norm_bounds(dtype, x64, w64, None, r64, factor, want, s64, saved)
    oo.assert_within("y", y[some.cuda()], want, e_y)
    oo.assert_within("s", s[some.cuda()], s64, e_s)
    dx, dr, dw = torch.autograd.grad([y, s], [x, r, w], [dy, ds])
    at = s.detach()[some.cuda()].cpu().double()
    here, _, saved = oo.norm(at, w64, None, 1e-5)
    e_h = oo.norm_bounds(dtype, at, w64, None, None, 1.0, here, at, saved)[2]
    h, q = saved
    g64 = dy64 * w64
    dr64 = q * (g64 - g64.mean(-1, keepdim=True) - h * (g64 * h).mean(-1, keepdim=True)) + ds64
    dx64 = oo.drop(dr64, kept[some], factor)
    bounds = oo.norm_backward_bounds(dtype, dy64, ds64, saved, w64, (dx64, dr64, torch.zeros(n), torch.zeros(n)), e_h, factor)
    oo.assert_within("dx", dx[some.cuda()], dx64, bounds[0])
    oo.assert_within("dr", dr[some.cuda()], dr64, bounds[1])
    a, b = new(40, 64) * 0.1, new(n, 40) * 0.1
    z = new(rows, 64)
    out = ops.low_rank_add(x.detach(), z, a, b)
    want, bound = oo.low_rank(dtype, x64, z[some.cuda()].cpu().double(), a.cpu().double()[None], b.cpu().double()[None], [1.0])["out"]
    oo.assert_within("out", out[some.cuda()], want, bound)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_long_batches(dtype):
    check_low_rank(4100, 512, 768, 16, dtype, flat=True)
    check_low_rank(2100, 256, 384, 64, dtype, 2, [0, 1000, 1003, 2090], [1, 0, 1])


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rank", [40, 64, 128])
def test_long_requests_of_high_rank(rank, dtype):
    # sums shared by workgroups and put together again, odd lengths of rows and of the last slab
    check_low_rank(2055, 1600, 900, rank, dtype, 2, [5, 900, 1003, 2049], [1, 0, 1])
    check_low_rank(2048, 1111, 1300, rank, dtype, flat=True)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_long_sums_of_high_rank(dtype):
    check_low_rank(2055, 8200, 300, 64, dtype, 2, [5, 900, 1003, 2049], [1, 0, 1])
    check_low_rank(2048, 300, 8193, 40, dtype, flat=True)
    check_low_rank(2100, 4101, 200, 128, dtype, flat=True)
    check_low_rank(2100, 200, 4097, 100, dtype, 2, [0, 130, 2000], [1, 0], scale=[0.5, 2.0])


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rank", [4, 8, 16, 32, 64, 128])
def test_single_tokens_in_one_launch_and_in_two(rank, dtype):
    """One launch makes both products while `in` is short enough, by the padded rank; in panels of several trips if `out` is long"""
    padded = max(rank, 16)
    border = (1 << 16) // (4 * padded) if dtype == torch.float32 else (1 << 18) // (2 * padded)
    starts = [1] + list(range(2, 41)) + [40, 42]
    which = [i % 4 - 1 for i in range(len(starts) - 1)]
    for k, n in ((border, 9000), (border + 1, 200), (min(border, 77), 4700)):
        check_low_rank(43, k, n, rank, dtype, 3, starts, which, scale=[0.5, -1.0, 2.0], step=n == 200 or k == 77)
        check_low_rank(2, k, n, rank, dtype, flat=True, step=n == 200)
    check_low_rank(43, 77, 4700, rank, dtype, 3, starts, which, inplace=True, step=False)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("k", [2, 3, 4, 5, 7, 8, 9, 15, 65, 130, 1027])
def test_ends_of_rows(k, dtype):
    """Short rows, and rows whose end is read with elements that were counted before: an infinity there counts once"""
    check_low_rank(37, k, 40, 12, dtype, flat=True)
    check_low_rank(2, k, 40, 8, dtype, flat=True, step=False)
    for rows in (1, 37):
        wide = torch.full((rows, k + 16), float("nan"), dtype=dtype, device="cuda")
        x = wide[:, 8:8 + k]
        x.fill_(1.0)
        x[:, max(k - 3, 0)] = float("inf")
        a, b = torch.ones(8, k, dtype=dtype, device="cuda"), torch.ones(24, 8, dtype=dtype, device="cuda")
        out = ops.low_rank_add(torch.zeros(rows, 24, dtype=dtype, device="cuda"), x, a, b)
        assert (out == float("inf")).all()


def test_single_tokens_of_more_requests_than_one_launch_takes():
    for tokens in (500, 520):
        check_low_rank(tokens, 72, 96, 16, torch.float16, 5, list(range(tokens + 1)), [i % 6 - 1 for i in range(tokens)])


def test_single_tokens_through_wide_layers():
    for rank in (1, 16, 64):
        check_low_rank(1, 8192, 8192, rank, torch.bfloat16, step=False, flat=True)
    check_low_rank(33, 4096, 1024, 16, torch.float16, 4, list(range(34)), [i % 5 - 1 for i in range(33)], step=False)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_low_rank_strides(dtype):
    check_low_rank(40, 200, 120, 8, dtype, cut=lambda t: t[:, 5:-4] if t.shape[1] > 100 else t)
    check_low_rank(40, 64, 64, 8, dtype, cut=lambda t: t[::2])
    check_low_rank(40, 40, 40, 8, dtype, cut=lambda t: t.t())


def test_adapters_on_rows_far_apart():
    """As the last tokens of long sequences are: the rows of x, y and dout 2^23 elements apart and a little more"""
    far = lambda t: torch.zeros(3, (1 << 23) + 8, dtype=t.dtype, device="cuda")[:, -64:].copy_(t) if t.is_cuda else t
    check_low_rank(3, 64, 64, 8, torch.bfloat16, cut=far)
    z = torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="in place"):
        ops.low_rank_add(far(z), z, z.new_zeros(8, 64), z.new_zeros(64, 8), inplace=True)


def test_a_sum_in_place_is_noticed_by_what_was_saved():
    x, a, b = torch.randn(5, 64, device="cuda"), torch.randn(8, 64, device="cuda"), torch.randn(64, 8, device="cuda")
    leaf = torch.randn(5, 64, device="cuda", requires_grad=True)
    y = torch.tanh(leaf)
    with torch.no_grad():
        assert ops.low_rank_add(y, x, a, b, inplace=True) is y
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    before = leaf.detach().clone()
    with pytest.raises(ValueError, match="leaf"):
        ops.low_rank_add(leaf, x, a, b, inplace=True)
    assert torch.equal(leaf.detach(), before)


@pytest.mark.parametrize("starts,which", [(None, None), ([2, 9, 30], [1, -1]), ([0, 35], [0])])
def test_the_sum_in_place_leaves_other_rows_alone(starts, which):
    check_low_rank(40, 64, 72, 8, torch.bfloat16, 1 if starts is None else 2, starts, which, inplace=True)
    if starts is None:
        return
    x, a, b = torch.randn(40, 64, device="cuda"), torch.randn(2, 8, 64, device="cuda"), torch.randn(2, 72, 8, device="cuda")
    y = torch.randn(40, 72, device="cuda")
    y[:2] = float("nan")
    y[36:] = float("inf")
    before = y.clone()
    s, w = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (starts, which)]
    for out in (ops.low_rank_add(y, x, a, b, starts=s, which=w), ops.low_rank_add(y, x, a, b, starts=s, which=w, inplace=True)):
        assert torch.equal(out[36:], before[36:])
        assert starts[0] == 0 or torch.isnan(out[:2]).all()


def test_rows_and_adapters_do_not_touch_each_other():
    # infinities and NaN in one request's rows, in an adapter that is not used, and in rows without a request
    x, x64 = normal((70, 96), torch.float16, 1)
    y, y64 = normal((70, 64), torch.float16, 2)
    a, a64 = normal((3, 8, 96), torch.float16, 3, 0.1)
    b, b64 = normal((3, 64, 8), torch.float16, 4, 0.3)
    starts, which = [0, 20, 21, 60], [0, 0, 1]
    want = oo.low_rank(torch.float16, y64, x64, a64, b64, [1.0] * 3, starts, which, y64)
    x[20] = float("nan")
    x[60:] = float("inf")
    a[2], b[2] = float("nan"), float("inf")
    x.requires_grad_(True)
    s, w = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (starts, which)]
    out = ops.low_rank_add(y, x, a, b, starts=s, which=w)
    others = [i for i in range(70) if i != 20]
    oo.assert_within("out", out[others], want["out"][0][others], want["out"][1][others])
    assert torch.isnan(out[20]).all()
    dx, = torch.autograd.grad(out, x, y)
    oo.assert_within("dx", dx, *want["dx"])


def test_low_rank_without_rows_or_requests():
    for dtype in TYPES:
        x, y = [torch.zeros(0, n, dtype=dtype, device="cuda", requires_grad=True) for n in (24, 16)]
        a, b = torch.ones(4, 24, dtype=dtype, device="cuda", requires_grad=True), torch.ones(16, 4, dtype=dtype, device="cuda", requires_grad=True)
        out = ops.low_rank_add(y, x, a, b)
        gx, ga, gb = torch.autograd.grad(out, (x, a, b), torch.zeros_like(out))
        assert gx.shape == (0, 24) and not ga.any() and not gb.any()
        check_low_rank(6, 24, 16, 4, dtype, 2, [0], [])


def test_low_rank_gradients_that_nobody_asks_for():
    x, a, b, y = [normal(s, torch.bfloat16, i)[0] for i, s in enumerate(((90, 64), (8, 64), (48, 8), (90, 48)))]
    dout = normal((90, 48), torch.bfloat16, 9)[0]
    for t in (x, a, b, y):
        t.requires_grad_(True)
    every = torch.autograd.grad(ops.low_rank_add(y, x, a, b), (x, a, b, y), dout)
    for i, leaf in enumerate((x, a, b, y)):
        for t in (x, a, b, y):
            t.requires_grad_(t is leaf)
        g, = torch.autograd.grad(ops.low_rank_add(y, x, a, b), leaf, dout)
        assert torch.equal(g, every[i])


def test_three_dimensions():
    x, a, b, y = [normal(s, torch.float32, i)[0] for i, s in enumerate(((3, 5, 64), (8, 64), (48, 8), (3, 5, 48)))]
    out = ops.low_rank_add(y, x, a, b)
    assert torch.equal(out.reshape(15, 48), ops.low_rank_add(y.reshape(15, 48), x.reshape(15, 64), a, b))


# ---- refusals that need tensors on a GPU -----------------------------------------------------------------------------

def test_refusals():
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    bad = [
        lambda: ops.dropout(z(3, 4), 1.5, 1),
        lambda: ops.dropout(z(3, 4), float("nan"), 1),
        lambda: ops.dropout(z(3, 4), 0.5, -1),
        lambda: ops.dropout(z(3, 4), 0.5, 1 << 64),
        lambda: ops.dropout(z(3, 4), 0.5, 1, call=-1),
        lambda: ops.dropout(z(3, 4), 0.5, i(1)),
        lambda: ops.dropout(z(3, 4), 0.5, torch.zeros(1, dtype=torch.int64)),
        lambda: ops.dropout(z(3, 4), 0.5, torch.zeros(2, dtype=torch.int64, device="cuda")),
        lambda: ops.dropout(z(), 0.5, 1),
        lambda: ops.dropout(z(3, 4), 0.5, 1, residual=z(3, 5)),
        lambda: ops.dropout(z(3, 4), 0.5, 1, residual=z(3, 4, dtype=torch.float16)),
        lambda: ops.dropout(z(3, 4), 0.5, 1, residual=torch.zeros(3, 4)),
        lambda: ops.layer_norm(z(3, 0)),
        lambda: ops.layer_norm(z(3, 4), z(5)),
        lambda: ops.layer_norm(z(3, 4), z(4), z(3, 4)),
        lambda: ops.layer_norm(z(3, 4), z(4, dtype=torch.bfloat16)),
        lambda: ops.layer_norm(z(3, 4), eps=-1e-5),
        lambda: ops.layer_norm(z(3, 4), p=0.1),
        lambda: ops.layer_norm(z(3, 4), residual=z(4, 4)),
        lambda: ops.low_rank_add(z(3, 4), z(2, 5), z(2, 5), z(4, 2)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 4), z(4, 2)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 5), z(4, 3)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(129, 5), z(4, 129)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 2, 5), z(3, 4, 2), starts=i(0, 3), which=i(0)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 2, 5), z(2, 4, 2)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 2, 5), z(2, 4, 2), starts=i(0, 3)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 2, 5), z(2, 4, 2), starts=i(0, 1, 3), which=i(0)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 2, 5), z(2, 4, 2), starts=i(0, 3).long(), which=i(0)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 2, 5), z(2, 4, 2), starts=i(0, 3).cpu(), which=i(0)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 5), z(4, 2), scale=z(2)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 5), z(4, 2), scale=z(1).half()),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 5), z(4, 2), scale=z(1).requires_grad_(True)),
        lambda: ops.low_rank_add(z(3, 4), z(3, 5), z(2, 5), z(4, 2), scale="2"),
        lambda: ops.low_rank_add(z(4, 3).t(), z(3, 5), z(2, 5), z(4, 2), inplace=True),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d is not refused" % n)
    with pytest.raises(ops.VmsError):       # rows that share memory cannot be written in place
        ops.low_rank_add(z(1, 4).expand(3, 4), z(3, 5), z(2, 5), z(4, 2), inplace=True)
