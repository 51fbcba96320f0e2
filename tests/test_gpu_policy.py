"""The policy with memory: frames -> first layer -> layer norm -> linear attention -> layer norm -> actions, acting and learning."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    assert _torch.cuda.is_available(), "these tests need the MI355X"
    return _torch


@pytest.fixture(scope="module")
def policy_module():
    from paper_2502_00021_amd import policy
    return policy


def _frames(torch, B, T, h=32, w=32):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    return torch.randint(0, 256, (B, T, 1, h, w, 3), generator=g, device="cuda", dtype=torch.uint8)


def test_acting_step_by_step_equals_the_rollout(torch, policy_module):
    """The same products in another order: a few roundings of bfloat16 (2^-8 each) between the two."""
    B, T = 12, 40
    policy = policy_module.MemoryPolicy(32, 32, 1, 5, width=64, heads=3, d_head=32)
    frames, resets = _frames(torch, B, T), torch.zeros((B, T), dtype=torch.bool, device="cuda")
    resets[3, 0] = resets[3, 17] = resets[5, 39] = True
    state = policy.first_state(B)
    acted = torch.stack([policy.act(frames[:, t].contiguous(), state, resets[:, t]) for t in range(T)], 1)
    with torch.no_grad():
        actions, last = policy(frames, resets)
    assert (acted - actions).square().mean().sqrt() <= 4 * 2.0 ** -8 * actions.square().mean().sqrt()
    assert (state - last).square().mean().sqrt() <= 4 * 2.0 ** -8 * last.square().mean().sqrt()
    # an episode that begins at step 17 sees nothing from before
    other = frames.clone()
    other[3, :17] = 255 - other[3, :17]
    with torch.no_grad():
        again, _ = policy(other, resets)
    assert not torch.equal(again[3, :17], actions[3, :17])
    assert (again[3, 17:] - actions[3, 17:]).abs().max() <= 2.0 ** -6 * actions.abs().max()


def test_gradients_through_both_operators(torch, policy_module):
    """Against the same composition in PyTorch's own float64 operations and autograd."""
    from paper_2502_00021_amd import pxr
    rng = np.random.default_rng(4)
    B, T, H, d = 3, 37, 2, 16
    ld = np.float32([-0.05, -0.7])
    layer = pxr.LinearAttention(H, d, d, ld)
    x = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((B, T, H * d), (H * d, 3 * H * d), (H * d,), (d,), (B, H, d, d))]
    resets = torch.from_numpy(rng.random((B, T)) < 0.1).cuda()
    weights = torch.from_numpy(rng.standard_normal((B, T, H, d))).cuda()
    weights_state = torch.from_numpy(rng.standard_normal((B, H, d, d))).cuda()

    def loss(x, w, n1, n2, s0, norm, attend):
        x = norm(x, n1)
        q, k, v = (p.unflatten(-1, (H, d)) for p in (x @ w).chunk(3, dim=-1))
        out, last = attend(q, k, v, s0)
        return (norm(out, n2) * weights.to(x.dtype)).sum() + (last * weights_state.to(x.dtype)).sum()

    def plain_norm(x, w):
        c = x - x.mean(-1, keepdim=True)
        return c * (c.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w

    def plain_attend(q, k, v, S):
        keep, outs = torch.exp(torch.from_numpy(ld).cuda().double())[None, :, None, None], []
        for t in range(T):
            S = torch.where(resets[:, t, None, None, None], 0.0, S * keep) + k[:, t, :, :, None] * v[:, t, :, None, :]
            outs.append((q[:, t, :, :, None] * S).sum(-2) * layer.scale)
        return torch.stack(outs, 1), S

    ours = [t.clone().requires_grad_() for t in x]
    loss(*ours, lambda x, w: policy_module.layer_norm(x, w), lambda q, k, v, s: policy_module.linear_attention(layer, q, k, v, resets, s)).backward()
    ref = [t.double().requires_grad_() for t in x]
    loss(*ref, plain_norm, plain_attend).backward()
    for a, b in zip(ours, ref):
        # fp32 throughout: sums of up to a thousand terms, each through two products and two normalisations
        assert (a.grad - b.grad).square().mean().sqrt() <= 2.0 ** -17 * b.grad.square().mean().sqrt()
    layer.close()


def test_learning_lowers_the_loss(torch, policy_module):
    B, T = 16, 24
    policy = policy_module.MemoryPolicy(32, 32, 1, 4, width=64, heads=2, d_head=32, seed=5)
    frames = _frames(torch, B, T)
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    target = torch.rand((B, T, 4), generator=g, device="cuda") - 0.5
    optimizer = torch.optim.Adam(policy.parameters(), lr=3e-3)
    losses = []
    for _ in range(25):
        loss = (policy(frames)[0] - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    assert all(p.grad is not None and bool(p.grad.isfinite().all()) for p in policy.parameters())
    assert losses[-1] < 0.5 * losses[0], losses


def test_what_is_written_in_place_between_forward_and_backward_is_noticed(torch, policy_module):
    """A state that goes on being stepped, a buffer that is written again, resets that change: the gradients would be those of the new values."""
    from paper_2502_00021_amd import pxr
    layer = pxr.LinearAttention(2, 16, 16, np.float32([-0.05, -0.7]))

    def start():
        x = [torch.ones((3, 20, 2, 16), device="cuda", requires_grad=True) for _ in range(3)]
        resets, state = torch.zeros((3, 20), dtype=torch.bool, device="cuda"), torch.ones((3, 2, 16, 16), device="cuda")
        return x, resets, state, policy_module.linear_attention(layer, *x, resets, state)[0]

    def step(x, resets, state):
        with torch.no_grad():
            layer.step(x[0][:, 0], x[1][:, 0], x[2][:, 0], state)

    def again(x, resets, state):
        layer.forward(x[0].detach(), x[1].detach(), x[2].detach(), state_out=state)

    def outputs(x, resets, state):
        layer.forward(*(t.detach().clone() for t in x), out=x[2].detach())

    def one_output(x, resets, state):
        layer.step(x[0].detach()[:, 0], x[1].detach()[:, 0], x[2].detach()[:, 0], state.clone(), out=x[0].detach()[:, 1])

    def mark(x, resets, state):
        resets[1, 3] = True
    start()[3].sum().backward()
    for write in (step, again, outputs, one_output, mark):
        x, resets, state, out = start()
        write(x, resets, state)
        with pytest.raises(RuntimeError, match="inplace"):
            out.sum().backward()
    # layer norm: its input written by each call that takes a buffer
    y = torch.randn((40, 64), device="cuda")
    _, mean, rstd = pxr.layer_norm(y)
    for write in (lambda x: pxr.layer_norm(y, out=x), lambda x: pxr.layer_norm_backward(y, y, mean, rstd, dx=x)):
        x = torch.randn((40, 64), device="cuda", requires_grad=True)
        out = policy_module.layer_norm(x)
        write(x.detach())
        with pytest.raises(RuntimeError, match="inplace"):
            out.sum().backward()
    layer.close()


def test_features_written_again_before_the_backward_pass_are_noticed(torch, policy_module):
    """The first layer's features in a buffer that the next step's take, normalised with a weight that learns."""
    from paper_2502_00021_amd import pxr
    conv = pxr.Conv(32, 32, 1, np.ones((3, 3, 3, 32), np.float32), np.zeros(32, np.float32))
    frames = _frames(torch, 4, 1)[:, 0].contiguous()
    features = conv.forward(frames)
    weight = torch.ones(features[0].numel(), device="cuda", requires_grad=True)
    out = policy_module.layer_norm(features.flatten(1), weight)
    conv.forward(frames, out=features)
    with pytest.raises(RuntimeError, match="inplace"):
        out.float().sum().backward()
    conv.close()
