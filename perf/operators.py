"""The operators of a training block that the framework offers (paper_2401_08156_amd/ops.py), as work to be measured.

Three kinds of cases: `dropout` (a mask from a counter-based generator, never stored), `layer_norm` (with the residual
sum and its dropout on the way in) and `low_rank` (adapters of many requests beside a shared projection).  A case's
values: `op`, `step` (forward and backward, or forward alone), `rows` x `cols` (tokens x features; `low_rank`: `rows`
tokens from `cols` to `out` features), `dtype`, `p` (share of elements dropped), `residual`, `affine` (has weights),
`rank`, `adapters`, `requests` (packed one behind the other, each with an adapter number or none; 0: one adapter for
all rows), `padding` (rows behind the last request).

A mask depends on the row, the column, a seed and the number of the call alone: Philox-4x32 with ten rounds (Salmon,
Moraes, Dror and Shaw, 2011) turns the counter (column / 8, row, call) under the key `seed` into eight 16-bit numbers,
and an element is kept where its number is at least p * 65536, rounded.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
CALL = (7 << 32) + 5        # number of the dropout call
SCALE = 0.5                 # of the adapters
MUL = (0xD2511F53, 0xCD9E8D57)
WEYL = (0x9E3779B9, 0xBB67AE85)
WORD = 0xFFFFFFFF


def _case(op, rows, cols, dtype, step, name=None, **more):
    c = dict(op=op, rows=rows, cols=cols, dtype=dtype, step=step, **more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the activations of the smallest training loop here (hidden 1024), forward and backward: launches count
        _case("dropout", 1024, 1024, "f32", True, p=0.1, residual=False, name="dropout-1024x1024-f32-step"),
        # odd sizes: a recomputed forward pass whose rows start at odd addresses
        _case("dropout", 777, 1001, "f16", False, p=0.25, residual=True, name="dropout-777x1001-f16"),
        # the four times wider activations of a recomputed layer of 4096 features
        _case("dropout", 4096, 16384, "bf16", True, p=0.1, residual=False, name="dropout-4096x16384-bf16-step"),
        # one token that a trained model answers with
        _case("layer_norm", 1, 4096, "bf16", False, p=0.0, residual=False, affine=True, name="norm-1x4096-bf16"),
        # the training loop on the live allocator: hidden 2048, no weights, residual
        _case("layer_norm", 2816, 2048, "f32", True, p=0.0, residual=True, affine=False, name="norm-2816x2048-f32-step"),
        # a sequence of odd length at the offloading workload's hidden size
        _case("layer_norm", 4099, 5120, "f16", True, p=0.0, residual=False, affine=True, name="norm-4099x5120-f16-step"),
        # four sequences of 4096 tokens of the recomputation workload: residual, dropout and weights
        _case("layer_norm", 16384, 4096, "bf16", True, p=0.1, residual=True, affine=True, name="norm-16384x4096-bf16-step"),
        # one token of one request
        _case("low_rank", 1, 4096, "bf16", False, out=4096, rank=16, adapters=1, requests=0, padding=0, name="lowrank-1-bf16"),
        # one token each of 96 requests, 32 adapters
        _case("low_rank", 96, 4096, "bf16", False, out=16384, rank=16, adapters=32, requests=96, padding=0, name="lowrank-96x1-bf16"),
        # prompts of 24 requests side by side, 12 adapters, a padded batch
        _case("low_rank", 6007, 4096, "f16", False, out=4096, rank=32, adapters=12, requests=24, padding=100, name="lowrank-24prompts-f16"),
        # the training loop on the live allocator with adapters
        _case("low_rank", 2560, 2048, "f32", True, out=8192, rank=8, adapters=1, requests=0, padding=0, name="lowrank-2560-f32-step"),
        # LoRA fine-tuning, the wide projection of a layer of 4096 features, the largest rank of the LoRA workload
        _case("low_rank", 8192, 4096, "bf16", True, out=16384, rank=64, adapters=1, requests=0, padding=0, name="lowrank-8192-bf16-step"),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("dropout", "layer_norm", "low_rank"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    step = rng.random() < 0.6
    while True:
        rows, cols = _spread(rng, 1, 16384), _spread(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        if op != "low_rank":
            if rows * cols > 1 << 26:
                continue
            p = rng.choice((0.0, 0.05, 0.1, 0.3, 0.5)) if op == "layer_norm" else rng.choice((0.05, 0.1, 0.3, 0.5))
            residual = rng.random() < 0.5
            if op == "dropout":
                return _case(op, rows, cols, dtype, step, p=p, residual=residual)
            return _case(op, rows, cols, dtype, step, p=p if residual else 0.0, residual=residual, affine=rng.random() < 0.7)
        out, rank = _spread(rng, 16, 16384), rng.choice((1, 4, 8, 12, 16, 16, 32, 64, 64, 100, 128))
        if rng.random() < 0.5:
            out = max(64, out // 64 * 64)
        requests = rng.choice((0, rows, _spread(rng, 1, 256)))
        if requests and rows < requests or requests > 1024:
            continue
        adapters = _spread(rng, 1, 32) if requests else 1
        if rows * (cols + out) > 1 << 27 or rows * (cols + out) * adapters * rank * (3 if step else 1) > 30e9:
            continue
        return _case(op, rows, cols, dtype, step, out=out, rank=rank, adapters=adapters, requests=requests,
                     padding=rows // 50 if 1 < requests < rows else 0)


def _lengths(case, seed):
    """Tokens of each request: a few long ones, many short ones, none empty."""
    n = case["requests"]
    free = case["rows"] - case["padding"] - n
    w = np.random.RandomState(seed % (1 << 31)).lognormal(0.0, 1.2, n)
    w = np.floor(w / w.sum() * free).astype(np.int64) + 1
    w[0] += case["rows"] - case["padding"] - w.sum()
    return w


def prepare(case, seed):
    t = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, by=1.0, around=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * by + around).to(t)

    s = dict(case=case, seed=(seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 64))
    m, k = case["rows"], case["cols"]
    s["x"] = normal(m, k)
    if case["op"] == "low_rank":
        n, r, out = case["adapters"], case["rank"], case["out"]
        one = case["requests"] == 0
        s["a"] = normal(*((r, k) if one else (n, r, k)), by=1 / math.sqrt(k))
        s["b"] = normal(*((out, r) if one else (n, out, r)), by=1 / math.sqrt(r))
        s["y"] = normal(m, out)
        s["starts"] = s["which"] = None
        if not one:
            lengths = _lengths(case, seed)
            which = np.random.RandomState(seed % (1 << 31) + 1).randint(-1 if n > 1 else 0, n, case["requests"])
            s["starts"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
            s["which"] = torch.from_numpy(which.astype(np.int32)).cuda()
        if case["step"]:
            s["dy"] = normal(m, out)
        leaves = ("x", "y", "a", "b")
    else:
        if case["p"]:
            s["words"] = _words(s["seed"])
        if case["residual"]:
            s["residual"] = normal(m, k)
        if case.get("affine"):
            s["weight"], s["bias"] = normal(k, by=0.1, around=1.0), normal(k, by=0.1)
        if case["step"]:
            s["dy"] = normal(m, k)
            if case["op"] == "layer_norm" and case["residual"]:
                s["ds"] = normal(m, k)
        leaves = ("x", "residual", "weight", "bias")
    if case["step"]:
        for name in leaves:
            if name in s:
                s[name].requires_grad_(True)
    return s


# ---- the framework's calls -------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2401_08156_amd import ops
    c = s["case"]
    with torch.set_grad_enabled(c["step"]):
        if c["op"] == "dropout":
            y = ops.dropout(s["x"], c["p"], s["seed"], CALL, residual=s.get("residual"))
        elif c["op"] == "layer_norm":
            y = ops.layer_norm(s["x"], s.get("weight"), s.get("bias"), EPS, residual=s.get("residual"), p=c["p"],
                               seed=s["seed"], call=CALL)
        else:
            y = ops.low_rank_add(s["y"], s["x"], s["a"], s["b"], SCALE, s["starts"], s["which"])
    y = y if isinstance(y, tuple) else (y,)
    if not c["step"]:
        return dict(zip(("y", "s"), y))
    names = [n for n in ("x", "residual", "weight", "bias", "a", "b") if n in s]
    grads = torch.autograd.grad(y, [s[n] for n in names], [s["dy"], s["ds"]] if len(y) > 1 else [s["dy"]])
    return dict(zip(("y", "s"), [v.detach() for v in y]), **{"d" + n: v for n, v in zip(names, grads)})


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ------------------------------------------

def _words(seed):
    """What the generator's rounds need beside the counter, on the GPU: factors, key, key step and number of the call."""
    pairs = [MUL, (seed & WORD, seed >> 32), WEYL, (CALL & WORD, CALL >> 32)]
    return torch.tensor(pairs, device="cuda").reshape(4, 2, 1, 1)


def _kept(rows, cols, p, words):
    """Truth values [rows, cols]: the 32-bit words in 64-bit integers, both products of a round side by side, the high
    half of each from the halves of its factor."""
    groups = (cols + 7) // 8
    by, key, step, call = words
    even = torch.zeros(2, rows, groups, dtype=torch.int64, device="cuda")
    even[0] += torch.arange(groups, device="cuda")
    even[1] += call[0]
    odd = torch.zeros_like(even)
    odd[0] += torch.arange(rows, device="cuda").unsqueeze(1)
    odd[1] += call[1]
    for _ in range(10):
        high = (by * (even >> 16) + (by * (even & 0xFFFF) >> 16)) >> 16
        even, odd = high.flip(0) ^ odd ^ key, (by * even & WORD).flip(0)
        key = key + step & WORD
    words = torch.stack([even[0], odd[0], even[1], odd[1]], dim=-1)
    u = torch.stack([words & 0xFFFF, words >> 16], dim=-1)
    return u.reshape(rows, -1)[:, :cols] >= math.floor(p * 65536 + 0.5)


def _factor(p):
    return 65536 / (65536 - math.floor(p * 65536 + 0.5))


def _run_dropout(s, c, t):
    f = _factor(c["p"])
    kept = _kept(c["rows"], c["cols"], c["p"], s["words"]) if c["p"] else None
    drop = (lambda v: torch.where(kept, v * f, 0.0)) if c["p"] else (lambda v: v)
    y = drop(s["x"].float())
    if c["residual"]:
        y = s["residual"].float() + y
    o = dict(y=y.to(t))
    if c["step"]:
        o["dx"] = drop(s["dy"].float()).to(t)
        if c["residual"]:
            o["dresidual"] = s["dy"]
    return o


def _run_norm(s, c, t):
    f = _factor(c["p"])
    kept = _kept(c["rows"], c["cols"], c["p"], s["words"]) if c["p"] else None
    drop = (lambda v: torch.where(kept, v * f, 0.0)) if c["p"] else (lambda v: v)
    v = drop(s["x"].float())
    if c["residual"]:
        v = s["residual"].float() + v
    d = v - v.mean(1, keepdim=True)
    q = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    h = d * q
    y = h * s["weight"].float() + s["bias"].float() if c["affine"] else h
    o = dict(y=y.to(t))
    if c["residual"]:
        o["s"] = v.to(t)
    if c["step"]:
        dy = s["dy"].float()
        g = dy * s["weight"].float() if c["affine"] else dy
        dv = q * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        if c["residual"]:
            dv = dv + s["ds"].float()
            o["dresidual"] = dv.to(t)
        o["dx"] = drop(dv).to(t)
        if c["affine"]:
            o["dweight"], o["dbias"] = (dy * h).sum(0).to(t), dy.sum(0).to(t)
    return o


def _run_low_rank(s, c, t):
    """All adapters side by side in two products; what a row's own adapter did not make is masked between them."""
    n, r, k, out, rows = c["adapters"], c["rank"], c["cols"], c["out"], c["rows"]
    x = s["x"].float()
    a = s["a"].float().reshape(n * r, k)
    b = s["b"].float().reshape(n, out, r).transpose(1, 2).reshape(n * r, out).contiguous()
    if c["requests"]:
        at = torch.searchsorted(s["starts"][1:], torch.arange(rows, dtype=torch.int32, device="cuda"), right=True)
        which = torch.cat([s["which"], s["which"].new_full((1,), -1)])[at]
        mask = (which.unsqueeze(1) == torch.arange(n, device="cuda")).repeat_interleave(r, dim=1) * SCALE
    else:
        mask = SCALE
    h = x @ a.t() * mask
    o = dict(y=(s["y"].float() + h @ b).to(t))
    if c["step"]:
        dy = s["dy"].float()
        dh = dy @ b.t() * mask
        o["dx"] = (dh @ a).to(t)
        o["da"] = (dh.t() @ x).reshape(s["a"].shape).to(t)
        o["db"] = (dy.t() @ h).reshape(out, n, r).transpose(0, 1).reshape(s["b"].shape).to(t).contiguous()
    return o


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    form = {"dropout": _run_dropout, "layer_norm": _run_norm, "low_rank": _run_low_rank}[c["op"]]
    with torch.no_grad():
        return form(state, c, DTYPES[c["dtype"]])


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    m, k = case["rows"], case["cols"]
    step = case["step"]
    if case["op"] == "low_rank":
        r, out = case["rank"], case["out"]
        used = min(case["adapters"], max(1, case["requests"])) * r * (k + out)
        # x, y, the weights read, the sum written; then dy and x read once more, dx and the weights' gradients written
        size = m * (k + 2 * out) + used + (m * (out + 2 * k) + 2 * used if step else 0)
        return {"bytes": e * size, "flops": 2 * m * r * (k + out) * (3 if step else 1)}
    tensors = 2 + case["residual"]
    if case["op"] == "dropout":
        tensors += 2 if step else 0                             # dy read, dx written; the residual's gradient is dy
        return {"bytes": e * tensors * m * k, "flops": 2 * m * k * (2 if step else 1)}
    tensors += case["residual"]                                 # the sum is written too
    if step:                                                    # dy and the sum read, the sum's own gradient, dx and dresidual
        tensors += 3 + case["residual"] + (1 if case["p"] else 0)
    return {"bytes": e * (tensors * m * k + (2 + 2 * step) * k * case["affine"]), "flops": (8 + 12 * step) * m * k}


# ---- the definition in 64 bits, row by row and request by request ----------------------------------------------------

def _kept_exact(rows, cols, p, seed):
    limit = int(math.floor(p * 65536 + 0.5))
    groups = -(-cols // 8)
    keep = np.empty((rows, groups * 8), dtype=bool)
    at_once = max(1, (1 << 18) // groups)
    m0, m1, word, half = np.uint64(MUL[0]), np.uint64(MUL[1]), np.uint64(WORD), np.uint64(32)
    for r0 in range(0, rows, at_once):
        r1 = min(rows, r0 + at_once)
        shape = (r1 - r0, groups)
        w0 = np.broadcast_to(np.arange(groups, dtype=np.uint64), shape)
        w1 = np.broadcast_to(np.arange(r0, r1, dtype=np.uint64)[:, None], shape)
        w2 = np.full(shape, CALL & WORD, dtype=np.uint64)
        w3 = np.full(shape, CALL >> 32, dtype=np.uint64)
        k0, k1 = seed & WORD, seed >> 32
        for _ in range(10):
            p0, p1 = w0 * m0, w2 * m1
            w0, w2 = (p1 >> half) ^ w1 ^ np.uint64(k0), (p0 >> half) ^ w3 ^ np.uint64(k1)
            w1, w3 = p1 & word, p0 & word
            k0, k1 = (k0 + WEYL[0]) & WORD, (k1 + WEYL[1]) & WORD
        both = np.stack([w0, w1, w2, w3], axis=-1).astype("<u4").view("<u2")
        keep[r0:r1] = (both >= limit).reshape(r1 - r0, groups * 8)
    return torch.from_numpy(keep[:, :cols].copy()).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    v = {k: t.detach().double() for k, t in s.items() if isinstance(t, torch.Tensor) and t.is_floating_point()}
    if case["op"] == "low_rank":
        return _exact_low_rank(case, seed, s, v)
    kept = _kept_exact(case["rows"], case["cols"], case["p"], s["seed"])
    factor = kept / (1.0 - math.floor(case["p"] * 65536 + 0.5) / 65536)
    total = v["x"] * factor + v.get("residual", 0.0)
    if case["op"] == "dropout":
        o = dict(y=total)
        if case["step"]:
            o["dx"] = v["dy"] * factor
            if case["residual"]:
                o["dresidual"] = v["dy"]
        return o
    var, mean = torch.var_mean(total, dim=1, correction=0, keepdim=True)
    sd = torch.sqrt(var + EPS)
    unit = (total - mean) / sd
    w, b = (v["weight"], v["bias"]) if case["affine"] else (1.0, 0.0)
    o = dict(y=unit * w + b)
    if case["residual"]:
        o["s"] = total
    if case["step"]:
        g = v["dy"] * w / sd
        ds = g - g.mean(1, keepdim=True) - unit * (unit * g).mean(1, keepdim=True) + v.get("ds", 0.0)
        o["dx"] = ds * factor
        if case["residual"]:
            o["dresidual"] = ds
        if case["affine"]:
            o["dweight"], o["dbias"] = (v["dy"] * unit).sum(0), v["dy"].sum(0)
    return o


def _exact_low_rank(case, seed, s, v):
    a, b = (w if w.dim() == 3 else w.unsqueeze(0) for w in (v["a"], v["b"]))
    if case["requests"]:
        ends = np.cumsum(_lengths(case, seed)).tolist()
        parts = list(zip([0] + ends[:-1], ends, s["which"].tolist()))
    else:
        parts = [(0, case["rows"], 0)]
    y = v["y"].clone()
    dx, da, db = torch.zeros_like(v["x"]), torch.zeros_like(a), torch.zeros_like(b)
    for lo, hi, k in parts:
        if k < 0:
            continue
        h = torch.mm(v["x"][lo:hi], a[k].t().contiguous())
        y[lo:hi] += SCALE * torch.mm(h, b[k].t().contiguous())
        if case["step"]:
            d = SCALE * v["dy"][lo:hi]
            dh = torch.mm(d, b[k])
            dx[lo:hi] = torch.mm(dh, a[k])
            da[k] += torch.mm(dh.t().contiguous(), v["x"][lo:hi])
            db[k] += torch.mm(d.t().contiguous(), h)
    if not case["step"]:
        return dict(y=y)
    return dict(y=y, dx=dx, da=da.reshape(s["a"].shape), db=db.reshape(s["b"].shape))
