"""A small policy with memory on the renderer's frames: what stands between the first convolutional layer and the actions.

    frames -> Conv (first layer) -> layer norm -> projection -> layer norm -> memory -> layer norm -> actions

The memory is one of three: `attention`, queries, keys and values through linear attention with a decay for each head; `turned`, the same
with queries and keys normalised for each head and turned by the step's position in its episode; `gated`, a gated recurrence, inputs
and gates from one projection.

Acting is one step of every environment (`act`: LinearAttention.step, gated_recurrence_step, the state updated in place); learning takes
whole rollouts with the episodes that begin inside them (`forward`, gradients by the operators' backward passes; a gradient
of a gradient is refused).  `Orthogonal` steps the weight matrices by orthogonalised updates.  The projections are matrix
products of PyTorch's.
`python -m paper_2502_00021_amd.policy [--memory turned|gated] [--orthogonal]` renders rollouts of the quadruped scene, acts on
them and learns from them."""
import argparse
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


class _HeadNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, layer, q, k, q_weight, k_weight, positions):
        ctx.layer = layer
        ctx.save_for_backward(q, k, q_weight, k_weight, positions)
        return layer.forward(q, k, q_weight, k_weight, positions=positions)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        q, k, q_weight, k_weight, positions = ctx.saved_tensors
        dq, dk = (None if x is None else d.contiguous() for x, d in ((q, dq), (k, dk)))
        dq, dk, dq_weight, dk_weight = ctx.layer.backward(dq, dk, q, k, q_weight, k_weight, positions=positions)
        return None, dq, dk, None if q_weight is None else dq_weight, None if k_weight is None else dk_weight, None


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, resets, state, coupled):
        ctx.coupled = coupled
        ctx.save_for_backward(x, gate, resets, state)
        ctx.set_materialize_grads(False)
        return pxr.gated_recurrence(x, gate, resets=resets, state=state, coupled=coupled)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        x, gate, resets, state = ctx.saved_tensors
        dout = torch.zeros_like(x, memory_format=torch.contiguous_format) if dout is None else dout.contiguous()
        dx, dgate, dstate = pxr.gated_recurrence_backward(dout, x, gate, resets=resets, state=state, coupled=ctx.coupled,
                                                          dstate=None if dlast is None else dlast.contiguous())
        return dx, dgate, None, dstate, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """pxr.layer_norm for torch.autograd: x [..., D] with adjacent values -> y; gradients for x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


def linear_attention(layer, q, k, v, resets=None, state=None):
    """LinearAttention.forward for torch.autograd: (out, the last state); gradients for q, k, v and the first state.  (The
    layer's decays are constants.)  A state that goes on being stepped is cloned first: the backward pass reads the one that
    was given, and raises where it has been written since."""
    return _LinearAttention.apply(layer, q, k, v, resets, state)


def head_norm(layer, q, k, q_weight=None, k_weight=None, positions=None):
    """HeadNorm.forward for torch.autograd: (q, k) normalised and turned (either may be None); gradients for q, k and the weights."""
    return _HeadNorm.apply(layer, q, k, q_weight, k_weight, positions)


def gated_recurrence(x, gate, resets=None, state=None, coupled=True):
    """pxr.gated_recurrence for torch.autograd: (out, the last state); gradients for x, gate and the first state.  A state that goes
    on being stepped is cloned first, as for linear_attention."""
    return _GatedRecurrence.apply(x, gate, resets, state, coupled)


def episode_positions(n_envs, n_steps, resets=None, first=None):
    """Steps since the episode began, int32 [B,T], for resets [B,T] (or None); first: int32 [B], the position of the first step where it
    begins no episode (0 unless given)."""
    at = torch.arange(n_steps, device="cuda", dtype=torch.int32).expand(n_envs, n_steps)
    goes_on = at if first is None else at + first[:, None]
    if resets is None:
        return goes_on.contiguous()
    began = torch.where(resets.bool(), at, -1).cummax(1).values
    return torch.where(began >= 0, at - began, goes_on)


class Orthogonal(torch.optim.Optimizer):
    """Steps weight matrices by their momentum with its singular values pushed towards one (pxr.orthogonalise), so that every direction
    of an update counts alike.  Matrices of one size and type go together.  Only matrices: vectors have no such update.  A matrix [m,n] with
    m > n takes lr * sqrt(m / n) of its update, the others lr of theirs.  Parameters are of the current device; a step that is refused has written nothing."""

    def __init__(self, params, lr=0.02, momentum=0.95, nesterov=True, steps=5, eps=1e-7):
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, steps=steps, eps=eps))
        for group in self.param_groups:
            for p in group["params"]:
                if p.dim() != 2:
                    raise ValueError(f"only matrices are orthogonalised, not {tuple(p.shape)}")

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        together = []
        for group in self.param_groups:
            same = {}
            for p in group["params"]:
                if p.grad is not None:
                    same.setdefault((p.shape, p.dtype, p.device), []).append(p)
            together += [(group, params) for params in same.values()]
        # (what a call refuses is refused here, before any momentum or parameter is another one)
        for group, params in together:
            pxr.orthogonalise_workspace(len(params), *params[0].shape, steps=group["steps"], eps=group["eps"])
            for p in params:
                if not (p.is_cuda and p.is_floating_point() and p.grad.layout == torch.strided):
                    raise ValueError(f"only dense gradients of real matrices on the GPU, not {p.dtype} {p.grad.layout} on {p.device}")
                pxr._here(torch, p)
        for group, params in together:
            updates = []
            for p in params:
                state = self.state[p]
                # (in fp32, whatever the parameter's type: also after torch has loaded it as of that type)
                m = state["momentum"].float() if "momentum" in state else torch.zeros(p.shape, dtype=torch.float32, device=p.device)
                state["momentum"] = m.mul_(group["momentum"]).add_(p.grad)
                updates.append(torch.add(p.grad, m, alpha=group["momentum"]).float() if group["nesterov"] else m)
            updates = pxr.orthogonalise(torch.stack(updates), steps=group["steps"], eps=group["eps"])
            # (a tall matrix has fewer directions than rows: the step of a row stays what it is for a square one)
            m, n = params[0].shape
            size = group["lr"] * max(1.0, m / n) ** 0.5
            for p, update in zip(params, updates):
                p.sub_(update, alpha=size)
        return loss


class MemoryPolicy(torch.nn.Module):
    """Actions from frame stacks [B,T,S,H,W,3] uint8 and a state per environment.  memory: "attention", "turned" or "gated" (its
    heads * d_head channels look back like the heads)."""

    def __init__(self, frame_h, frame_w, n_stack, n_actions, width=256, heads=4, d_head=64, seed=0, memory="attention"):
        super().__init__()
        if memory not in ("attention", "turned", "gated"):
            raise ValueError(f"memory is attention, turned or gated, not {memory!r}")
        rng = np.random.default_rng(seed)
        self.conv = pxr.Conv(frame_h, frame_w, n_stack, (rng.standard_normal((3, 3, 3 * n_stack, 32)) * 0.15).astype(np.float32),
                             np.zeros(32, np.float32))
        features = self.conv.Ho * self.conv.Wo * 32
        # the heads look back over 8 to 512 steps
        windows = 2.0 ** np.linspace(3, 9, heads)
        self.kind, self.heads, self.d_head = memory, heads, d_head
        parts = 2 if memory == "gated" else 3
        if memory == "gated":
            # a gate of log(w - 1) keeps 1 - 1 / w
            self.bias_gate = torch.nn.Parameter(torch.from_numpy(np.log(np.repeat(windows, d_head) - 1)).float().cuda())
        else:
            self.memory = pxr.LinearAttention(heads, d_head, d_head, np.log1p(-1 / windows).astype(np.float32))
        if memory == "turned":
            self.turn = pxr.HeadNorm(d_head)
            self.norm_q, self.norm_k = (torch.nn.Parameter(torch.ones(d_head, device="cuda")) for _ in range(2))

        def matrix(n, m):
            return torch.nn.Parameter((torch.from_numpy(rng.standard_normal((n, m))).float() / math.sqrt(n)).cuda())
        self.w_in, self.w_qkv, self.w_out = matrix(features, width), matrix(width, parts * heads * d_head), matrix(heads * d_head, n_actions)
        self.norm_in, self.norm_heads = (torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (width, d_head))
        self.bias_in = torch.nn.Parameter(torch.zeros(width, device="cuda"))

    def close(self):
        for layer in ("conv", "memory", "turn"):
            if hasattr(self, layer):
                getattr(self, layer).close()

    def first_state(self, n_envs):
        """Before an episode; `turned`: (the state, int32 [B] the position of the next step)."""
        if self.kind == "gated":
            return torch.zeros((n_envs, self.heads * self.d_head), device="cuda")
        state = torch.zeros((n_envs, self.heads, self.d_head, self.d_head), device="cuda")
        return (state, torch.zeros(n_envs, dtype=torch.int32, device="cuda")) if self.kind == "turned" else state

    def _parts(self, frames):
        """[N,S,H,W,3] -> queries, keys, values [N, heads, d_head], or inputs and gates [N, heads * d_head] (parts of one projection), bfloat16."""
        x = layer_norm(self.conv.forward(frames).flatten(1))  # no gradient: the first layer's weights are constants
        x = layer_norm(x @ self.w_in.bfloat16(), self.norm_in, self.bias_in)
        x = x @ self.w_qkv.bfloat16()
        if self.kind == "gated":
            x, gate = x.chunk(2, dim=-1)
            return x, gate + self.bias_gate.bfloat16()
        return (p.unflatten(-1, (self.heads, self.d_head)) for p in x.chunk(3, dim=-1))

    def _actions(self, seen):
        """[..., heads, d_head] -> [..., n_actions] float32."""
        return (layer_norm(seen, self.norm_heads).flatten(-2) @ self.w_out.bfloat16()).float()

    def forward(self, frames, resets=None, state=None):
        """A rollout: frames [B,T,S,H,W,3], resets [B,T], state as of first_state or None (a clone, if `act` takes the same one before the
        backward pass) -> actions [B,T,n], the last state."""
        B, T = frames.shape[:2]
        parts = [x.unflatten(0, (B, T)) for x in self._parts(frames.flatten(0, 1))]
        if self.kind == "gated":
            seen, last = gated_recurrence(*parts, resets, state)
            return self._actions(seen.unflatten(-1, (self.heads, self.d_head))), last
        if self.kind == "attention":
            seen, last = linear_attention(self.memory, *parts, resets, state)
            return self._actions(seen), last
        q, k, v = parts
        state, first = (None, None) if state is None else state
        positions = episode_positions(B, T, resets, first)
        q, k = head_norm(self.turn, q, k, self.norm_q, self.norm_k, positions)
        seen, last = linear_attention(self.memory, q, k, v, resets, state)
        return self._actions(seen), (last, positions[:, -1] + 1)

    @torch.no_grad()
    def act(self, frames, state, resets=None):
        """One step: frames [B,S,H,W,3]; state is updated in place -> actions [B,n]."""
        parts = self._parts(frames)
        if self.kind == "gated":
            seen = pxr.gated_recurrence_step(*parts, state, resets=resets)
            return self._actions(seen.unflatten(-1, (self.heads, self.d_head)))
        if self.kind == "attention":
            return self._actions(self.memory.step(*parts, state, resets=resets))
        q, k, v = parts
        state, position = state
        if resets is not None:
            position.masked_fill_(resets.bool(), 0)
        q, k = self.turn.forward(q, k, self.norm_q, self.norm_k, positions=position)
        seen = self.memory.step(q, k, v, state, resets=resets)
        position.add_(1)
        return self._actions(seen)


def main(n_envs=64, n_steps=48, updates=30, memory="attention", orthogonal=False):
    from paper_2502_00021_amd import workloads
    w = workloads.make(3, B=n_envs)
    scene = pxr.Scene(w["desc"])
    scene.apply_distractor(dict(w["distractor"]))
    policy = MemoryPolicy(scene.H, scene.W, 1, n_actions=8, memory=memory)
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
    if memory == "turned":
        state, last = state[0], last[0]
    print(f"{n_envs} environments, {n_steps} steps: acted step by step and as a rollout, largest difference "
          f"{float((acted - actions).abs().max()):.3g} of {float(actions.abs().max()):.3g}; states {float((state - last).abs().max()):.3g}")
    # learning: actions that depend on what was seen some steps ago
    target = torch.tanh(acted.roll(5, 1)) * 0.5
    if orthogonal:
        matrices = [p for p in policy.parameters() if p.dim() == 2]
        optimizers = [Orthogonal(matrices, lr=0.004), torch.optim.Adam([p for p in policy.parameters() if p.dim() != 2], lr=3e-3)]
    else:
        optimizers = [torch.optim.Adam(policy.parameters(), lr=3e-3)]
    for i in range(updates):
        loss = (policy(frames, resets)[0] - target).square().mean()
        for optimizer in optimizers:
            optimizer.zero_grad()
        loss.backward()
        for optimizer in optimizers:
            optimizer.step()
        if i % 10 == 0 or i + 1 == updates:
            print(f"update {i}: loss {float(loss.detach()):.4f}", flush=True)
    policy.close()
    scene.close()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--memory", choices=("attention", "turned", "gated"), default="attention")
    ap.add_argument("--orthogonal", action="store_true", help="step the weight matrices by orthogonalised updates")
    a = ap.parse_args()
    main(memory=a.memory, orthogonal=a.orthogonal)
