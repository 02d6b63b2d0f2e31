"""The operators' boundary without a GPU: the oracle's pins, declarations against exports, and every refusal of the C
entry points and of the Python functions (none of which launches anything)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import ops_oracle as oo
from paper_2401_08156_amd import binding, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESTRUCT, EWORKSPACE = -1, -2, -4


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vms_ops.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(vms_[a-z0-9_]+)\s*\(", text))) == sorted(ops.EXPORTS)
    for n in ops.EXPORTS:
        assert hasattr(ops.lib(), n)


def test_struct_layouts_match_the_header():
    sizes = dict(vms_dropout_mask=32, vms_dropout_args=104, vms_layernorm_args=152, vms_layernorm_backward_args=184,
                 vms_lowrank_args=152, vms_lowrank_backward_args=224)
    for n, size in sizes.items():
        assert ctypes.sizeof(getattr(ops, n)) == size, n


@pytest.mark.parametrize("counter,key,words", [
    # the generator's published known answers (Salmon, Moraes, Dror and Shaw, 2011)
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_the_oracles_generator_gives_the_published_numbers(counter, key, words):
    assert tuple(oo.philox(counter, key)) == words


def test_the_oracles_numbers_are_the_generators_by_row_and_column():
    seed, call = 0x299F31D0A4093822, (9 << 32) + 4
    n = oo.numbers(3, 21, seed, call)
    for t, c in ((0, 0), (0, 7), (0, 8), (1, 9), (2, 20), (2, 15)):
        w = oo.philox((c // 8, t, 4, 9), (seed & 0xFFFFFFFF, seed >> 32))[c % 8 // 2]
        assert n[t, c] == (w >> 16 if c % 2 else w & 0xFFFF)


def test_a_share_p_of_the_oracles_elements_is_dropped():
    # 2^20 independent elements: six standard deviations of the share are 6 sqrt(p (1 - p) / 2^20)
    for p in (0.1, 0.5):
        kept, factor = oo.mask((1024, 1024), p, 77, 3)
        assert abs(float((~kept).double().mean()) - p) < 6 * (p * (1 - p) / 2 ** 20) ** 0.5 + 2 ** -17
        assert abs(factor * (1 - p) - 1) < 2 ** -15


def test_the_oracles_gradients_are_those_of_differences():
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    x, res, w, b, dy, ds = r(4, 9), r(4, 9), r(9), r(9), r(4, 9), r(4, 9)

    def f(x, res, w, b):
        y, s, _ = oo.norm(x, w, b, 1e-3, res, 0.25, 5, 6)
        return (y * dy).sum() + (s * ds).sum()
    _, _, saved = oo.norm(x, w, b, 1e-3, res, 0.25, 5, 6)
    grads = oo.norm_backward(dy, ds, saved, w, x.shape, 0.25, 5, 6)
    for i, want in zip((0, 1, 2, 3), grads):
        args = [x, res, w, b]
        d, e = r(*args[i].shape), 1e-6
        lo, hi = list(args), list(args)
        lo[i], hi[i] = args[i] - e * d, args[i] + e * d
        # the difference quotient's error: e^2 of the third derivative and 2^-53 of f over e
        assert abs(float((f(*hi) - f(*lo)) / (2 * e) - (want * d).sum())) < 1e-7

    y, x, a, b, dout = r(7, 5), r(7, 6), r(2, 3, 6), r(2, 5, 3), r(7, 5)
    parts = dict(starts=[0, 2, 2, 6], which=[1, 0, 0])

    def f(x, a, b):
        return (oo.low_rank(torch.float32, y, x, a, b, [0.5, 2.0], **parts)["out"][0] * dout).sum()
    got = oo.low_rank(torch.float32, y, x, a, b, [0.5, 2.0], dout=dout, **parts)
    for i, n in enumerate(("dx", "da", "db")):
        args = [x, a, b]
        d, e = r(*args[i].shape), 1e-6
        lo, hi = list(args), list(args)
        lo[i], hi[i] = args[i] - e * d, args[i] + e * d
        assert abs(float((f(*hi) - f(*lo)) / (2 * e) - (got[n][0] * d).sum())) < 1e-7


# ---- refusals of the C entry points: addresses that nothing follows, since no call below gets to a launch ------------

P = 1 << 20


def dropout_args(**kw):
    a = ops.vms_dropout_args(104, ops.VMS_BF16, 4, 16, P, None, P, 16, 16, 16, ops.vms_dropout_mask(0.1, 1, None, 0))
    return changed(a, kw)


def norm_args(**kw):
    a = ops.vms_layernorm_args(152, ops.VMS_F32, 4, 16, P, P, P, P, P, P, P, 16, 16, 16, 16, 1e-5, ops.vms_dropout_mask(0.1, 1, None, 0))
    return changed(a, kw)


def norm_backward_args(**kw):
    a = ops.vms_layernorm_backward_args(184, ops.VMS_F32, 4, 16, P, P, P, P, P, P, P, P, P, 16, 16, 16, 16, 16,
                                        ops.vms_dropout_mask(0.1, 1, None, 0), P, 1 << 20)
    return changed(a, kw)


def lowrank_args(**kw):
    a = ops.vms_lowrank_args(152, ops.VMS_F16, 40, 64, 32, 8, 3, 5, 1.0, None, P, P, P, P, P, P, P, 64, 32, 32, P, 1 << 30)
    return changed(a, kw)


def lowrank_backward_args(f=None, **kw):
    a = ops.vms_lowrank_backward_args(224, 0, lowrank_args(**(f or {})), P, P, P, P, 32, 64, P, 1 << 30)
    return changed(a, kw)


def changed(a, kw):
    for k, v in kw.items():
        where = a
        if k in ("p", "d_seed"):
            where = a.mask
        assert hasattr(where, k)
        setattr(where, k, v)
    return a


@pytest.mark.parametrize("name,make,kw,code", [
    *[("vms_dropout", dropout_args, kw, code) for kw, code in [
        (dict(struct_size=8), ESTRUCT), (dict(dtype=3), EINVAL), (dict(rows=1 << 31), EINVAL), (dict(cols=1 << 31), EINVAL),
        (dict(p=-0.1), EINVAL), (dict(p=1.5), EINVAL), (dict(p=float("nan")), EINVAL), (dict(d_seed=P + 4), EINVAL),
        (dict(d_x=None), EINVAL), (dict(d_y=None), EINVAL), (dict(d_x=P + 1), EINVAL), (dict(d_residual=P + 1), EINVAL),
        (dict(ldy=15), EINVAL), (dict(ldx=1 << 31), EINVAL)]],
    *[("vms_layernorm", norm_args, kw, code) for kw, code in [
        (dict(struct_size=8), ESTRUCT), (dict(dtype=9), EINVAL), (dict(cols=0), EINVAL), (dict(cols=1 << 26), EINVAL), (dict(rows=1 << 40), EINVAL),
        (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(p=2.0), EINVAL), (dict(d_x=None), EINVAL),
        (dict(d_y=P + 2), EINVAL), (dict(d_residual=None), EINVAL), (dict(d_residual=None, p=0.0), EINVAL),
        (dict(d_weight=P + 2), EINVAL), (dict(d_stats=P + 2), EINVAL), (dict(ldy=8), EINVAL), (dict(lds=8), EINVAL)]],
    *[("vms_layernorm_backward", norm_backward_args, kw, code) for kw, code in [
        (dict(struct_size=8), ESTRUCT), (dict(dtype=3), EINVAL), (dict(cols=0), EINVAL), (dict(d_dy=None), EINVAL),
        (dict(d_s=None), EINVAL), (dict(d_stats=None), EINVAL), (dict(d_dres=None), EINVAL), (dict(d_dweight=P + 2), EINVAL),
        (dict(lddx=4), EINVAL), (dict(d_workspace=None), EWORKSPACE), (dict(d_workspace=P + 4), EWORKSPACE),
        (dict(workspace_bytes=127), EWORKSPACE)]],
    *[("vms_lowrank", lowrank_args, kw, code) for kw, code in [
        (dict(struct_size=8), ESTRUCT), (dict(dtype=3), EINVAL), (dict(rows=1 << 28), EINVAL), (dict(in_=0), EINVAL),
        (dict(out=1 << 22), EINVAL), (dict(rank=0), EINVAL), (dict(rank=129), EINVAL), (dict(n_adapters=0), EINVAL),
        (dict(n_adapters=65536), EINVAL), (dict(n_requests=1 << 16), EINVAL), (dict(rows=(1 << 28) - 1, n_requests=1 << 15, out=(1 << 22) - 1, rank=5, ldy=1 << 22, ldo=1 << 22, d_out=2 * P, hidden_bytes=1 << 50), EINVAL), (dict(d_x=None), EINVAL), (dict(d_a=None), EINVAL),
        (dict(d_b=P + 1), EINVAL), (dict(d_y=None), EINVAL), (dict(d_out=None), EINVAL), (dict(ldo=31), EINVAL),
        (dict(d_which=None), EINVAL), (dict(d_starts=P + 2), EINVAL), (dict(ldy=64), EINVAL), (dict(d_hidden=None), EWORKSPACE),
        (dict(d_hidden=P + 4), EWORKSPACE), (dict(hidden_bytes=64), EWORKSPACE),
        # (more workgroups than a launch can have, of either product)
        (dict(rows=1 << 27, rank=128, n_requests=1, d_out=2 * P, hidden_bytes=1 << 50), EINVAL)]],
    *[("vms_lowrank_backward", lowrank_backward_args, kw, code) for kw, code in [
        (dict(struct_size=8), ESTRUCT), (dict(f=dict(struct_size=8)), ESTRUCT), (dict(f=dict(rank=200)), EINVAL),
        (dict(f=dict(d_x=None)), EINVAL), (dict(f=dict(d_hidden=None)), EWORKSPACE), (dict(d_dout=None), EINVAL),
        (dict(d_da=P + 1), EINVAL), (dict(lddx=63), EINVAL), (dict(d_workspace=None), EWORKSPACE), (dict(workspace_bytes=100), EWORKSPACE),
        (dict(f=dict(rows=1 << 27, rank=128, n_requests=1, hidden_bytes=1 << 50), workspace_bytes=1 << 50), EINVAL)]],
])
def test_the_c_entry_points_refuse(name, make, kw, code):
    assert getattr(ops.lib(), name)(ctypes.byref(make(**kw)), None) == code


def test_null_arguments_and_calls_without_rows():
    L = ops.lib()
    for n in ops.EXPORTS:
        assert getattr(L, n)(*([None] if n.endswith("_bytes") else [None, None])) == (0 if n.endswith("_bytes") else EINVAL)
    # nothing to do: no pointer is looked at, nothing is launched
    assert L.vms_dropout(ctypes.byref(dropout_args(rows=0, d_x=None, d_y=None)), None) == 0
    assert L.vms_dropout(ctypes.byref(dropout_args(cols=0, d_x=None, d_y=None)), None) == 0
    assert L.vms_layernorm(ctypes.byref(norm_args(rows=0, d_x=None, d_y=None)), None) == 0
    assert L.vms_layernorm_backward(ctypes.byref(norm_backward_args(rows=0, d_dweight=None, d_dbias=None)), None) == 0
    assert L.vms_lowrank(ctypes.byref(lowrank_args(rows=0, d_x=None, d_y=None, d_out=None)), None) == 0
    assert L.vms_lowrank_backward(ctypes.byref(lowrank_backward_args(f=dict(rows=0), d_da=None, d_db=None)), None) == 0


def test_workspaces_go_by_the_gradients_that_are_asked_for():
    L = ops.lib()
    ln = lambda **kw: L.vms_layernorm_backward_workspace_bytes(ctypes.byref(norm_backward_args(**kw)))
    assert ln(d_dweight=None, d_dbias=None) == 0 and ln() == 2 * 16 * 4 and ln(d_dbias=None) == ln()
    lr = lambda **kw: L.vms_lowrank_backward_workspace_bytes(ctypes.byref(lowrank_backward_args(**kw)))
    assert lr() > lr(d_da=None) > lr(d_da=None, d_dx=None) > 0
    assert lr(f=dict(rows=0)) == 0 and lr(f=dict(rank=0)) == 0
    assert L.vms_lowrank_hidden_bytes(ctypes.byref(lowrank_args())) >= 40 * 16 * 4
    assert L.vms_lowrank_hidden_bytes(ctypes.byref(lowrank_args(rank=0))) == 0
    assert L.vms_lowrank_hidden_bytes(ctypes.byref(lowrank_args(rows=0))) == 0


# ---- refusals of the Python functions ----------------------------------------------------------------------------------

@pytest.mark.parametrize("call", [
    lambda x: ops.dropout(x, 0.1, 1),
    lambda x: ops.layer_norm(x),
    lambda x: ops.low_rank_add(x, x, x, x),
])
def test_tensors_off_the_gpu_and_other_types_are_refused(call):
    with pytest.raises(ValueError, match="GPU"):
        call(torch.zeros(4, 4))
    with pytest.raises(ValueError, match="float32"):
        call(torch.zeros(4, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="float32"):
        call(torch.zeros(4, 4, dtype=torch.float64))


def test_the_binding_has_no_other_path():
    assert binding.lib() is ops.lib()
    import subprocess
    needed = subprocess.run(["readelf", "-d", ops._build.EXT], stdout=subprocess.PIPE, text=True).stdout
    assert "[libvmsreplay.so]" in needed and ops.nodes().__file__ == ops._build.EXT


@pytest.mark.parametrize("make,same,stride", [
    (lambda: torch.zeros(5, 8), True, 8),
    (lambda: torch.zeros(5, 16)[:, 3:11], True, 16),
    (lambda: torch.zeros(8).expand(5, 8), True, 0),
    (lambda: torch.zeros(5, 8, 2)[..., 0], False, 8),
    (lambda: torch.zeros(8, 5).t(), False, 8),
    (lambda: torch.zeros(2, 3, 8), True, 8),
    (lambda: torch.zeros(2, 3, 16)[..., :8], True, 16),
    (lambda: torch.zeros(2, 4, 8)[:, :3], False, 8),
    (lambda: torch.zeros(1, 4, 8)[:, :3], True, 8),
    (lambda: torch.zeros(()).expand(2, 3, 8), False, 8),
    (lambda: torch.zeros(3, 2, 8).transpose(0, 1), False, 8),
    (lambda: torch.zeros(8), True, 8),
    (lambda: torch.zeros(16)[::2], False, 8),
    (lambda: torch.zeros(1, 1, 16)[..., :8], True, 8),
    (lambda: torch.zeros(5, 1), True, 1),
    (lambda: torch.zeros(5, 7)[:, 2:3], True, 7),
])
def test_rows_of_any_strides(make, same, stride):
    t = make()
    m, ld = ops.nodes().matrix(t)
    assert (m is t) == same and ld == stride
    cols = t.size(-1)
    rows = t.numel() // cols
    flat = torch.as_strided(m, (rows, cols), (ld, 1), m.storage_offset())
    assert torch.equal(flat, t.reshape(rows, cols)) and flat.shape == t.reshape(rows, cols).shape


def test_rows_too_far_apart_for_the_library_are_copied():
    for apart, same in (((1 << 31) - 1, True), (1 << 31, False)):
        t = torch.empty(apart + 8, dtype=torch.int8).as_strided((2, 8), (apart, 1))     # (memory that nothing touches is not taken)
        t[0], t[1] = torch.arange(8), torch.arange(8, 16)
        m, ld = ops.nodes().matrix(t)
        assert (m is t) == same and ld == (apart if same else 8) and torch.equal(m, torch.arange(16, dtype=torch.int8).reshape(2, 8))


@pytest.mark.parametrize("module,argv", [
    ("torch_plugin", ["--dropout", "0.1"]), ("torch_plugin", ["--strategy", "X"]), ("torch_plugin", ["--strategy", "N", "--dropout", "2"]),
    ("torch_plugin", ["--strategy", "L", "--rank", "0"]), ("trace_import", ["--text", "nothing.txt", "--strategy", "L"]),
    ("trace_import", ["--record", "--dropout", "0.5"]),
])
def test_the_commands_refuse_options_that_do_not_go_together(module, argv, monkeypatch, capsys):
    import importlib
    import sys
    monkeypatch.setattr(sys, "argv", [module] + argv)
    with pytest.raises(SystemExit) as e:
        importlib.import_module("paper_2401_08156_amd." + module).main()
    assert e.value.code == 2 and "--" in capsys.readouterr().err
