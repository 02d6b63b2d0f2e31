"""The live stitching allocator as PyTorch's device allocator for a whole process (the paper's
artefact is such a plug-in, Sec. 4.3), on a small training loop whose tensor sizes change every step.

    python -m paper_2401_08156_amd.torch_plugin            # every device allocation goes through vms_live
    python -m paper_2401_08156_amd.torch_plugin --native   # PyTorch's own caching allocator, for comparison
    python -m paper_2401_08156_amd.torch_plugin --strategy LR --dropout 0.1     # LoRA and recomputation

--strategy names the memory-saving strategies (the paper's Fig. 10) that the loop trains with: N none, R
recomputation of every block in the backward pass, L low-rank adapters on frozen weights, LR both.  The block is then
the one of block() below, made of the operators of ops.py.

The allocator has to be installed before the process touches device memory, hence one process per
mode.  Prints one JSON line: step time, loss of the last step, reserved / active peaks and, for the
plug-in, its decision counts and the time spent in the driver's virtual-memory calls.
"""
import argparse
import json
import time


def install():
    import torch
    from . import binding
    alloc = binding.torch_pluggable_allocator()
    torch.cuda.memory.change_current_allocator(alloc)
    return alloc


STRATEGIES = ("N", "R", "L", "LR")


def make_layer(hidden, strategy, rank, dev):
    """The tensors of one block; those that are trained require a gradient."""
    import torch
    new = lambda *shape: torch.randn(shape, device=dev)
    layer = dict(w=new(hidden, 4 * hidden) * 0.02, v=new(4 * hidden, hidden) * 0.02,
                 weight=torch.ones(hidden, device=dev), bias=torch.zeros(hidden, device=dev))
    trained = ["weight", "bias"]
    if "L" in strategy:
        layer.update(a1=new(rank, hidden) * hidden ** -0.5, b1=torch.zeros(4 * hidden, rank, device=dev),
                     a2=new(rank, 4 * hidden) * (4 * hidden) ** -0.5, b2=torch.zeros(hidden, rank, device=dev))
        trained += ["a1", "b1", "a2", "b2"]
    else:
        trained += ["w", "v"]
    for name in trained:
        layer[name].requires_grad_(True)
    return layer


def block(x, layer, number, dropout, seed, scale=2.0):
    """x = norm(x + drop(down(drop(gelu(up(x)))))), with adapters beside up and down where the layer has them.  The masks
    go by `seed` and the layer's number, so a block that is computed again drops the same elements."""
    import torch
    from . import ops
    u = x @ layer["w"]
    if "a1" in layer:
        u = ops.low_rank_add(u, x, layer["a1"], layer["b1"], scale, inplace=True)
    u = torch.nn.functional.gelu(u)
    if dropout:
        u = ops.dropout(u, dropout, seed, 2 * number)
    f = u @ layer["v"]
    if "a2" in layer:
        f = ops.low_rank_add(f, u, layer["a2"], layer["b2"], scale, inplace=True)
    return ops.layer_norm(f, layer["weight"], layer["bias"], residual=x, p=dropout, seed=seed, call=2 * number + 1)[0]


def train(steps, hidden, layers, seed=0, on_step=None, strategy=None, dropout=0.0, rank=16):
    """An MLP stack with recomputation-like reuse: the batch x sequence extent changes every step."""
    import torch
    from torch.utils.checkpoint import checkpoint
    if strategy is not None and strategy not in STRATEGIES:
        raise ValueError("strategy is one of %s, got %r" % (", ".join(STRATEGIES), strategy))
    if strategy is None and dropout:
        raise ValueError("dropout needs a strategy")
    torch.manual_seed(seed)
    dev = torch.device("cuda:0")
    if strategy is None:
        ws = [(torch.randn(hidden, 4 * hidden, device=dev) * 0.02).requires_grad_(True) for _ in range(layers)]
        vs = [(torch.randn(4 * hidden, hidden, device=dev) * 0.02).requires_grad_(True) for _ in range(layers)]
        trained = ws + vs
    else:
        stack = [make_layer(hidden, strategy, rank, dev) for _ in range(layers)]
        trained = [t for layer in stack for t in layer.values() if t.requires_grad]
    times, loss = [], None
    for i in range(steps):
        tokens = 1024 + 256 * ((i * 7) % 13)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        x = torch.randn(tokens, hidden, device=dev)
        if strategy is None:
            for w, v in zip(ws, vs):
                x = torch.nn.functional.layer_norm(x + torch.nn.functional.gelu(x @ w) @ v, (hidden,))
        else:
            for n, layer in enumerate(stack):
                args = (x, layer, n, dropout, (seed * steps + i) % (1 << 64))
                x = checkpoint(block, *args, use_reentrant=False) if "R" in strategy else block(*args)
        loss = (x[:, :8] ** 2).mean()
        loss.backward()
        with torch.no_grad():
            for p in trained:
                p -= 1e-3 * p.grad
                p.grad = None
        torch.cuda.synchronize()
        times.append(time.perf_counter() - t0)
        if on_step:
            on_step(i)
    return times, float(loss.detach())


def add_strategy_options(ap):
    ap.add_argument("--strategy", choices=STRATEGIES, help="memory-saving strategies to train with")
    ap.add_argument("--dropout", type=float, default=0.0, help="share of the activations that is dropped (with --strategy)")
    ap.add_argument("--rank", type=int, default=16, help="rank of the adapters (strategies L and LR)")


def strategy_options(ap, args):
    """The options as arguments of train()."""
    if args.dropout and not args.strategy:
        ap.error("--dropout needs --strategy")
    if not 0.0 <= args.dropout <= 1.0:
        ap.error("--dropout is a share from 0 to 1")
    if not 1 <= args.rank <= 128:
        ap.error("--rank is from 1 to 128")
    return dict(strategy=args.strategy, dropout=args.dropout, rank=args.rank)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--native", action="store_true")
    ap.add_argument("--steps", type=int, default=78)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--threshold", type=int, default=None, help="StitchFree threshold (cached sBlocks)")
    add_strategy_options(ap)
    args = ap.parse_args()
    strategy = strategy_options(ap, args)
    new_blocks = []                 # sBlocks created so far, after every step
    on_step = None
    if not args.native:
        import os
        if args.threshold is not None:
            os.environ["VMS_LIVE_SPOOL_THRESHOLD"] = str(args.threshold)
        install()
        from . import binding
        on_step = lambda i: new_blocks.append(int(binding.torch_allocator_stats(0)[0]["n_sblock_created"]))
    import torch
    times, loss = train(args.steps, args.hidden, args.layers, on_step=on_step, **strategy)
    half = len(times) // 2
    out = dict(mode="native" if args.native else "vms_live", steps=args.steps, loss=loss,
               ms_per_step_first_half=1e3 * sum(times[:half]) / half,
               ms_per_step_second_half=1e3 * sum(times[half:]) / (len(times) - half))
    if args.strategy:
        out.update(strategy)
    if args.native:
        out["peak_reserved_mib"] = torch.cuda.max_memory_reserved() / 2 ** 20
        out["peak_active_mib"] = torch.cuda.max_memory_allocated() / 2 ** 20
    else:
        from . import binding
        st, api = binding.torch_allocator_stats(0)
        out["peak_reserved_mib"] = int(st["peak_reserved"]) / 2 ** 20
        out["peak_active_mib"] = int(st["peak_active"]) / 2 ** 20
        out["fragmentation"] = float(st["fragmentation"])
        out["decisions"] = dict(exact=int(st["n_code"][1]), split=int(st["n_code"][2]), stitch=int(st["n_code"][3]),
                                grow=int(st["n_code"][4]), oom=int(st["n_code"][5]), free=int(st["n_code"][0]))
        out["sblocks_created"] = int(st["n_sblock_created"])
        period = 13                 # the token counts repeat every 13 steps
        out["sblocks_created_per_period"] = [new_blocks[min(k + period, len(new_blocks)) - 1] - (new_blocks[k - 1] if k else 0)
                                             for k in range(0, len(new_blocks), period)]
        out["sblocks_released"] = int(st["n_sblock_evicted"])
        out["driver_ms"] = dict(create=api.ms_create, map=api.ms_map, set_access=api.ms_set_access,
                                reserve=api.ms_reserve, unmap=api.ms_unmap)
        out["malloc_calls"] = int(api.n_malloc)
        out["ms_in_malloc"] = api.ms_malloc
    print(json.dumps(out))


if __name__ == "__main__":
    main()
