"""Calls of the operators that are refused before a tensor's device matters, and the build."""
import pytest
import torch

from paper_2401_08156_amd import ops

CALLS = [
    lambda x: ops.dropout(x, 0.5, 1),
    lambda x: ops.dropout(torch.zeros(4, 8), 0.5, 1, residual=x),
    lambda x: ops.layer_norm(x),
    lambda x: ops.layer_norm(torch.zeros(4, 8), x[0]),
    lambda x: ops.low_rank_add(x, x, x[:2], x[:, :2]),
    lambda x: ops.low_rank_add(torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(2, 8), x[:, :2]),
]


@pytest.mark.parametrize("call", CALLS)
def test_forward_mode_gradients_are_refused(call):
    import torch.autograd.forward_ad as forward
    x = torch.ones(4, 8)
    with forward.dual_level():
        with pytest.raises(ValueError, match="forward-mode"):
            call(forward.make_dual(x, x))
        with pytest.raises(ValueError, match="GPU"):        # no tangent, no refusal for it
            call(x)


@pytest.mark.parametrize("call", CALLS)
def test_traces_are_refused(call):
    from torch.fx.experimental.proxy_tensor import make_fx
    x = torch.ones(4, 8)
    with pytest.raises(ValueError, match="traced"):
        torch.jit.trace(call, x)
    for kw in (dict(), dict(tracing_mode="fake"), dict(tracing_mode="symbolic"), dict(pre_dispatch=True)):
        with pytest.raises(ValueError, match="traced"):
            make_fx(call, **kw)(x)
    with pytest.raises(ValueError, match="GPU"):            # what was refused leaves nothing behind
        call(x)


@pytest.mark.parametrize("there", [True, False])
def test_the_library_builds_without_pytorch(there, monkeypatch, capsys):
    """(what is run is looked at, nothing is compiled)"""
    import sys
    from paper_2401_08156_amd import build
    commands = []
    monkeypatch.setattr(build, "_run", lambda cmd, cwd: commands.append(cmd) or "")
    if not there:
        monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build(force=True) == build.LIB
    made = [c[c.index("-o") + 1] for c in commands]
    assert build.LIB in made and (build.EXT in made) == there
    compiled = [c[c.index("-c") + 1].split("/")[-1] for c in commands if "-c" in c]
    assert sorted(compiled) == sorted(build.SOURCES + build.OPS_SOURCES + [build.EXT_SOURCE] * there)
    assert not there or made.index(build.LIB) < made.index(build.EXT)
    assert ("no PyTorch" in capsys.readouterr().out) != there
    # what is there already is enough
    monkeypatch.setattr(build, "EXT", build.EXT if there else build.EXT + ".none")
    newest = max(build.os.path.getmtime(f) for f in (build.LIB, build.EXT) if build.os.path.exists(f))
    monkeypatch.setattr(build.os.path, "getmtime", lambda f: newest + (f in (build.LIB, build.EXT)))
    assert not build._stale()


def test_a_failed_compilation_is_told(monkeypatch):
    from paper_2401_08156_amd import build
    with pytest.raises(RuntimeError, match="g\\+\\+ failed"):
        build._run(["g++", "no_such_file.cpp"], build.CSRC)
