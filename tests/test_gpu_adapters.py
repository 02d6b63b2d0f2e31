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
