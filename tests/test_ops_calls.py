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
