"""The policy's operators under PyTorch's autograd, on the CPU: stand-ins in PyTorch's own operations take the kernels' place."""
import pytest
import torch

from paper_2502_00021_amd import policy


def _layer_norm(x, weight=None, bias=None, eps=1e-5):
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    y = (x - mean) * rstd * (1 if weight is None else weight) + (0 if bias is None else bias)
    return y, mean[..., 0], rstd[..., 0]


def _layer_norm_backward(dy, x, mean, rstd, weight=None):
    xh = (x - mean[..., None]) * rstd[..., None]
    g = dy * (1 if weight is None else weight)
    dx = rstd[..., None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


class _Layer:
    """Attention that looks at its own step alone: out = (q . k) v."""

    def forward(self, q, k, v, resets=None, state=None):
        return (q * k).sum(-1, keepdim=True) * v, torch.zeros(()) if state is None else state.clone()

    def backward(self, dout, q, k, v, resets=None, state=None, dstate=None):
        along = (dout * v).sum(-1, keepdim=True)
        return along * k, along * q, dout * (q * k).sum(-1, keepdim=True), dstate


@pytest.fixture
def stand_ins(monkeypatch):
    monkeypatch.setattr(policy.pxr, "layer_norm", _layer_norm)
    monkeypatch.setattr(policy.pxr, "layer_norm_backward", _layer_norm_backward)
    return _Layer()


def _inputs(*shapes):
    g = torch.Generator()
    g.manual_seed(1)
    return [torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True) for s in shapes]


def test_gradients(stand_ins):
    x, w, b = _inputs((5, 12), (12,), (12,))
    assert torch.autograd.gradcheck(lambda *a: policy.layer_norm(*a), (x, w, b))
    q, k, v = _inputs(*[(2, 3, 1, 4)] * 3)
    assert torch.autograd.gradcheck(lambda *a: policy.linear_attention(stand_ins, *a)[0], (q, k, v))


def test_a_gradient_of_a_gradient_is_refused(stand_ins):
    """There are no kernels for it: a penalty on a gradient must not be left out without a word."""
    x, w = _inputs((5, 12), (12,))
    y = policy.layer_norm(x, w)
    dx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (y.sum() + dx.square().sum()).backward()
    q, k, v = _inputs(*[(2, 3, 1, 4)] * 3)
    out = policy.linear_attention(stand_ins, q, k, v)[0]
    dq, = torch.autograd.grad(out.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (out.sum() + dq.square().sum()).backward()


def test_resets_that_change_between_forward_and_backward_are_noticed(stand_ins):
    q, k, v = _inputs(*[(2, 3, 1, 4)] * 3)
    resets = torch.zeros((2, 3), dtype=torch.bool)
    out = policy.linear_attention(stand_ins, q, k, v, resets)[0]
    resets[0, 1] = True
    with pytest.raises(RuntimeError, match="inplace"):
        out.sum().backward()
