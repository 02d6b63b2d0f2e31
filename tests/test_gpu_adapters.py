"""Low-rank adapters at the sizes that choose a variant of their own, against the oracle in 64 bits."""
import pytest
import torch

import ops_oracle as oo
from paper_2401_08156_amd import ops
from test_gpu_ops import TYPES, ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rank,length", [(16, None), (64, None), (100, None), (40, 1000), (16, 100), (128, 90)])
def test_sums_larger_than_the_last_cache(rank, length, dtype):
    """y and out, or dx, take more than 256 MiB: accesses marked as not to be kept, with tiles of 128 rows (one request, or long
    ones, up to rank 64) and of 64.  The oracle sees the first and last rows of tiles and requests."""
    e = torch.finfo(dtype).bits // 8
    rows, n = 4203, 32808 // e
    k = 80 if length else 65608 // e
    assert rows * n * e * 2 > 256 << 20 and (length or rows * k * e > 256 << 20)
    g = torch.Generator(device="cuda").manual_seed(rank)
    new = lambda *s, by=1.0: (torch.randn(s, generator=g, device="cuda") * by).to(dtype)
    starts = None if length is None else list(range(2, rows - 1, length)) + [rows - 1]
    which = None if length is None else [i % 4 - 1 for i in range(len(starts) - 1)]
    adapters = 1 if length is None else 3
    x, y, a, b = new(rows, k), new(rows, n), new(adapters, rank, k, by=k ** -0.5), new(adapters, n, rank, by=rank ** -0.5)
    i32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")
    edges = {0, 15, 16, 31, 32, 63, 64, 127, 128, 129, rows // 2, rows - 2, rows - 1}
    for s in (starts or [])[:6] + (starts or [])[-3:]:
        edges |= {s - 1, s, s + 63, s + 64}
    some = sorted(r for r in edges if 0 <= r < rows)
    # the sampled rows as a batch of their own
    if starts is None:
        few = None
    else:
        few = [sum(r < s for r in some) for s in starts]
    pick = lambda t: t.detach()[torch.tensor(some, device="cuda")].cpu().double()
    dout = new(rows, n) if length is None else None
    want = oo.low_rank(dtype, pick(y), pick(x), a.cpu().double(), b.cpu().double(), [0.5] * adapters, few, which, pick(dout) if length is None else None)
    args = dict(scale=0.5, starts=i32(starts), which=i32(which))
    if length is None:
        x.requires_grad_(True)
    out = ops.low_rank_add(y, x, a, b, **args) if adapters > 1 else ops.low_rank_add(y, x, a[0], b[0], 0.5)
    oo.assert_within("out", pick(out), *want["out"])
    if length is None:
        dx, = torch.autograd.grad(out, x, dout)
        oo.assert_within("dx", pick(dx), *want["dx"])
    with torch.no_grad():
        before = out.detach().clone()
        y2 = ops.low_rank_add(y, x, a if adapters > 1 else a[0], b if adapters > 1 else b[0], **args, inplace=True)
        assert y2 is y and torch.equal(y, before)


def one_of_each_column(rows, cols, dtype, seed):
    """a matrix with one number in each column, in a row of its own choice; (on the GPU, in 64 bits)"""
    g = torch.Generator().manual_seed(seed)
    v = torch.zeros(rows, cols, dtype=torch.float64)
    v[torch.randint(0, rows, (cols,), generator=g), torch.arange(cols)] = torch.randn(cols, generator=g, dtype=torch.float64)
    v = v.to(dtype)
    return v.cuda(), v.double()


def product(dtype, n, h, e_h, v):
    """How far h v may be off, rounded to the type, where every element of it is one product (of n that are summed): h by e_h and
    by what two values of the type leave of it (u of the first, u of that by the second), the product by its roundings in 32 bits"""
    u, chain = oo.unit(dtype), (n / 4 + oo.DEPTH) * oo.EMMA
    e = e_h + (0.0 if dtype == torch.float32 else u * u * (h.abs() + e_h) + oo.tiny(dtype))
    want, off = h @ v, e @ v.abs() + chain * ((h.abs() + e) @ v.abs())
    return want, u * want.abs() + (1 + u) * off + oo.tiny(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,rank,tokens", [(3, 16, False), (37, 8, False), (700, 128, False), (1100, 64, False), (2300, 32, False), (5000, 16, False), (2100, 64, False),
                                              (40, 16, True), (300, 64, True), (600, 128, True)])
def test_hidden_values_are_not_rounded_to_the_type(rows, rank, tokens, dtype):
    """x a^T and dout b are sums in 32 bits; the products that read them round once, to their outputs, in batches of every size.
    With one number in each column of b, dout, a or x every output is one product, so that a rounding in between would show."""
    k, n, scale = (4200 if rows == 2100 else 96), 160, 0.5
    normal = lambda *s, seed: (lambda t: (t.cuda(), t.double()))(torch.randn(s, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(dtype))
    starts = torch.arange(rows + 1, dtype=torch.int32, device="cuda") if tokens else None
    which = torch.zeros(rows, dtype=torch.int32, device="cuda") if tokens else None

    def run(x, a, b, dout):
        leaves = [t[None] if i and tokens else t for i, t in enumerate((x, a, b))]
        for t in leaves:
            t.requires_grad_(True)
        out = ops.low_rank_add(torch.zeros(rows, b.shape[0], dtype=dtype, device="cuda"), *leaves, scale=scale, starts=starts, which=which)
        return out, [g.reshape(t.shape) for g, t in zip(torch.autograd.grad(out, leaves, dout), (x, a, b))]
    hidden = lambda v, w: (scale * (v @ w.t()), ((v.shape[1] / 4 + oo.DEPTH) * oo.EMMA + 2 * oo.E32) * abs(scale) * (v.abs() @ w.abs().t()))
    # hidden = scale x a^T through b and dout
    (x, x64), (a, a64) = normal(rows, k, seed=1), normal(rank, k, seed=2)
    (bt, bt64), (dout, dout64) = one_of_each_column(rank, n, dtype, 3), one_of_each_column(rows, n, dtype, 4)
    h, e_h = hidden(x64, a64)
    out, (_, _, db) = run(x, a, bt.t().contiguous(), dout)
    oo.assert_within("out", out, *product(dtype, rank, h, e_h, bt64))
    oo.assert_within("db", db.t(), *product(dtype, rows, h.t(), e_h.t(), dout64))
    # dhidden = scale dout b through a and x
    (dout, dout64), (b, b64) = normal(rows, n, seed=5), normal(n, rank, seed=6)
    (a, a64), (x, x64) = one_of_each_column(rank, k, dtype, 7), one_of_each_column(rows, k, dtype, 8)
    h, e_h = hidden(dout64, b64.t())
    _, (dx, da, _) = run(x, a, b, dout)
    oo.assert_within("dx", dx, *product(dtype, rank, h, e_h, a64))
    oo.assert_within("da", da, *product(dtype, rows, h.t(), e_h.t(), x64))
