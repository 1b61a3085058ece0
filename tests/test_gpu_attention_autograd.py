"""attention under autograd: what it keeps where no graph is made."""
import pytest
import torch

from paper_2609_04910_amd import attention as at

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
def test_nothing_is_kept_without_a_graph(off, monkeypatch):
    """The part of out that its rounding leaves is for the backward pass: not written, and no memory
    taken, under no_grad, though the inputs require gradients."""
    q, k, v = (torch.randn((2, 300, 4, 64), device="cuda").half().requires_grad_() for _ in range(3))
    lows, fwd = [], at._fwd
    monkeypatch.setattr(at, "_fwd", lambda *args: lows.append(args[6]) or fwd(*args))
    want = at.attention(q, k, v, causal=True)
    assert lows[0] is not None and want.requires_grad
    torch.autograd.grad(want.float().sum(), (q, k, v))
    with off():
        out = at.attention(q, k, v, causal=True)
        assert at.attention(q.detach(), k.detach(), v.detach(), causal=True).equal(out)
    assert lows[1] is None and lows[2] is None and not out.requires_grad
    assert torch.equal(out, want.detach())
