"""A small policy with memory on the renderer's frames: what stands between the first convolutional layer and the actions.

    frames -> Conv (first layer) -> layer norm -> projection -> layer norm -> queries, keys, values
           -> linear attention with a decay for each head -> layer norm of each head -> actions

Acting is one step of every environment (`act`, LinearAttention.step, the state updated in place); learning takes whole
rollouts with the episodes that begin inside them (`forward`, gradients by LinearAttention.backward and
layer_norm_backward; a gradient of a gradient is refused).  The projections are matrix products of PyTorch's.
`python -m paper_2502_00021_amd.policy` renders rollouts of the quadruped scene, acts on them and learns from them."""
import math

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from paper_2502_00021_amd import pxr


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = pxr.layer_norm(x, weight, bias, eps=eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.biased = bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dweight, dbias = pxr.layer_norm_backward(dy.contiguous(), x, mean, rstd, weight)
        return dx, dweight if weight is not None else None, dbias if ctx.biased else None, None


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, layer, q, k, v, resets, state):
        out, last = layer.forward(q, k, v, resets=resets, state=state)
        ctx.layer = layer
        ctx.save_for_backward(q, k, v, resets, state)
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        q, k, v, resets, state = ctx.saved_tensors
        dout = torch.zeros_like(v, memory_format=torch.contiguous_format) if dout is None else dout.contiguous()
        dq, dk, dv, dstate = ctx.layer.backward(dout, q, k, v, resets=resets, state=state,
                                                dstate=None if dlast is None else dlast.contiguous())
        return None, dq, dk, dv, None, dstate


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """pxr.layer_norm for torch.autograd: x [..., D] with adjacent values -> y; gradients for x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


def linear_attention(layer, q, k, v, resets=None, state=None):
    """LinearAttention.forward for torch.autograd: (out, the last state); gradients for q, k, v and the first state.  (The
    layer's decays are constants.)  A state that goes on being stepped is cloned first: the backward pass reads the one that
    was given, and raises where it has been written since."""
    return _LinearAttention.apply(layer, q, k, v, resets, state)


class MemoryPolicy(torch.nn.Module):
    """Actions from frame stacks [B,T,S,H,W,3] uint8 and a state per environment."""

    def __init__(self, frame_h, frame_w, n_stack, n_actions, width=256, heads=4, d_head=64, seed=0):
        super().__init__()
        rng = np.random.default_rng(seed)
        self.conv = pxr.Conv(frame_h, frame_w, n_stack, (rng.standard_normal((3, 3, 3 * n_stack, 32)) * 0.15).astype(np.float32),
                             np.zeros(32, np.float32))
        features = self.conv.Ho * self.conv.Wo * 32
        # the heads look back over 8 to 512 steps
        windows = 2.0 ** np.linspace(3, 9, heads)
        self.memory = pxr.LinearAttention(heads, d_head, d_head, np.log1p(-1 / windows).astype(np.float32))
        self.heads, self.d_head = heads, d_head

        def matrix(n, m):
            return torch.nn.Parameter((torch.from_numpy(rng.standard_normal((n, m))).float() / math.sqrt(n)).cuda())
        self.w_in, self.w_qkv, self.w_out = matrix(features, width), matrix(width, 3 * heads * d_head), matrix(heads * d_head, n_actions)
        self.norm_in, self.norm_heads = (torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (width, d_head))
        self.bias_in = torch.nn.Parameter(torch.zeros(width, device="cuda"))

    def first_state(self, n_envs):
        return torch.zeros((n_envs, self.heads, self.d_head, self.d_head), device="cuda")

    def _qkv(self, frames):
        """[N,S,H,W,3] -> queries, keys, values [N, heads, d_head] (parts of one projection), bfloat16."""
        x = layer_norm(self.conv.forward(frames).flatten(1))  # no gradient: the first layer's weights are constants
        x = layer_norm(x @ self.w_in.bfloat16(), self.norm_in, self.bias_in)
        return (p.unflatten(-1, (self.heads, self.d_head)) for p in (x @ self.w_qkv.bfloat16()).chunk(3, dim=-1))

    def _actions(self, seen):
        """[..., heads, d_head] -> [..., n_actions] float32."""
        return (layer_norm(seen, self.norm_heads).flatten(-2) @ self.w_out.bfloat16()).float()

    def forward(self, frames, resets=None, state=None):
        """A rollout: frames [B,T,S,H,W,3], resets [B,T], state [B,heads,d,d] or None (a clone, if `act` takes the same one before the
        backward pass) -> actions [B,T,n], the last state."""
        B, T = frames.shape[:2]
        q, k, v = (x.unflatten(0, (B, T)) for x in self._qkv(frames.flatten(0, 1)))
        seen, last = linear_attention(self.memory, q, k, v, resets, state)
        return self._actions(seen), last

    @torch.no_grad()
    def act(self, frames, state, resets=None):
        """One step: frames [B,S,H,W,3]; state is updated in place -> actions [B,n]."""
        return self._actions(self.memory.step(*self._qkv(frames), state, resets=resets))


def main(n_envs=64, n_steps=48, updates=30):
    from paper_2502_00021_amd import workloads
    w = workloads.make(3, B=n_envs)
    scene = pxr.Scene(w["desc"])
    scene.apply_distractor(dict(w["distractor"]))
    policy = MemoryPolicy(scene.H, scene.W, 1, n_actions=8)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    resets = torch.rand((n_envs, n_steps), generator=g, device="cuda") < 1 / 24
    poses = torch.from_numpy(w["poses"]).cuda()
    frames = torch.empty((n_envs, n_steps, 1, scene.H, scene.W, 3), dtype=torch.uint8, device="cuda")
    state, acted = policy.first_state(n_envs), []
    for t in range(n_steps):  # acting: render, one step of the memory
        frames[:, t] = scene.render_batch(poses, step0=t)[0]
        acted.append(policy.act(frames[:, t].contiguous(), state, resets[:, t]))
    acted = torch.stack(acted, 1)
    with torch.no_grad():
        actions, last = policy(frames, resets)
    print(f"{n_envs} environments, {n_steps} steps: acted step by step and as a rollout, largest difference "
          f"{float((acted - actions).abs().max()):.3g} of {float(actions.abs().max()):.3g}; states {float((state - last).abs().max()):.3g}")
    # learning: actions that depend on what was seen some steps ago
    target = torch.tanh(acted.roll(5, 1)) * 0.5
    optimizer = torch.optim.Adam(policy.parameters(), lr=3e-3)
    for i in range(updates):
        loss = (policy(frames, resets)[0] - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        if i % 10 == 0 or i + 1 == updates:
            print(f"update {i}: loss {float(loss.detach()):.4f}", flush=True)
    policy.conv.close()
    policy.memory.close()
    scene.close()


if __name__ == "__main__":
    main()
