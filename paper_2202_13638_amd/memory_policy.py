"""A policy with memory, made of the library's block join, gated recurrence or linear attention, layer norm, clipping and AdamW: for machines of which
not every state is measured.

A stack of recurrent blocks over the steps of recorded trajectories, packed one after the other.  With R(z) = z / sqrt(mean(z^2) + eps),
per block

    [value | forget | gate] = y W_in^T,   h = recurrence(value, forget + bias),   z = h W_out^T,
    x <- x + scale * silu(gate) * (R(z) * post),   y = R(x) * pre,

from x = observations W_obs^T to actions = y W_act^T.  With ``heads`` the memory is a matrix for every head instead of a number for every channel:

    [query | key | value | gate] = y W_in^T,   h = layer norm of every head of attention(query, key, value), z = h W_out^T,

with a decay for every head that is its constant.  Dense products are torch's; everything between them is one call of the library
each.  Trained on whole trajectories (``forward``, ``backward``, ``update``), used one control period at a time (``start``, ``step``).

``python -m paper_2202_13638_amd.memory_policy`` records rollouts of a memoryless policy that sees all states and trains one with memory to act
like it from the positions alone.
"""
from __future__ import annotations

from typing import Dict, List, Optional

import torch

from . import binding

EPS = 1e-6


class MemoryPolicy:
    """Parameters are float32; matrices have a working copy in the type of the activations, which the update writes in the same pass."""

    def __init__(self, d_in: int, d_out: int, width: int, blocks: int, dtype=torch.bfloat16, state_bits: int = 32, seed: int = 0, heads: int = 0):
        g = torch.Generator().manual_seed(seed)
        self.width, self.blocks, self.dtype, self.seed, self.updates = width, blocks, dtype, seed, 0
        if heads < 0 or heads and (width % heads or width // heads > binding.ATTENTION_MAX_WIDTH):
            raise ValueError(f"heads must divide the width, into parts of {binding.ATTENTION_MAX_WIDTH} at most")
        self.memory = _Heads(width, heads) if heads else _Channels(width)

        def matrix(rows, columns):
            return (torch.randn(rows, columns, generator=g) / columns ** 0.5).cuda()

        def vector(value):
            return torch.full((width,), value, device="cuda")

        self.matrices: Dict[str, torch.Tensor] = {"obs": matrix(width, d_in), "act": matrix(d_out, width)}
        self.vectors: Dict[str, torch.Tensor] = {"pre0": vector(1.0)}
        for i in range(blocks):
            self.matrices[f"in{i}"], self.matrices[f"out{i}"] = matrix(self.memory.columns + width, width), matrix(width, width)
            self.vectors.update(self.memory.vectors(i))
            self.vectors.update({f"post{i}": vector(1.0), f"scale{i}": vector(0.5), f"pre{i + 1}": vector(1.0)})
        self.work = {k: m.to(dtype) for k, m in self.matrices.items()}
        self.moments = {k: _Moments(p, state_bits) for k, p in {**self.matrices, **self.vectors}.items()}

    # ------------------------------------------------------------------------------------------------ whole trajectories
    def forward(self, observations: torch.Tensor, offsets, initial: Optional[List[torch.Tensor]] = None):
        """Actions for observations[rows, d_in] of packed trajectories (see bagel_recurrence for `offsets`), and what backward() needs."""
        v, w = self.vectors, self.work
        obs = observations.to(self.dtype)
        x = obs @ w["obs"].t()
        y = torch.empty_like(x)
        binding.bagel_block_join(None, x, None, y, pre_weight=v["pre0"], eps=EPS)
        kept = {"obs": obs, "offsets": offsets, "initial": initial, "x": [x], "y": [y], "proj": [], "h": [], "z": [], "memory": []}
        for i in range(self.blocks):
            proj = y @ w[f"in{i}"].t()
            gate = proj[:, self.memory.columns:]
            h, of_memory = self.memory.forward(proj, v, i, offsets, initial[i] if initial else None)
            z = h @ w[f"out{i}"].t()
            x_in, x, y = x, torch.empty_like(x), torch.empty_like(x)
            binding.bagel_block_join(z, x_in, x, y, gate=gate, act="silu", post_weight=v[f"post{i}"], scale=v[f"scale{i}"],
                                     pre_weight=v[f"pre{i + 1}"], eps=EPS)
            for key, t in (("x", x), ("y", y), ("proj", proj), ("h", h), ("z", z), ("memory", of_memory)):
                kept[key].append(t)
        return y @ w["act"].t(), kept

    def backward(self, kept, d_actions: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Gradients of all parameters for the gradient of the actions."""
        v, w = self.vectors, self.work
        d_actions = d_actions.to(self.dtype)
        grads = {k: torch.empty_like(p) for k, p in self.vectors.items()}
        grads["act"] = d_actions.t() @ kept["y"][-1]
        dy, dx = d_actions @ w["act"], None
        for i in reversed(range(self.blocks)):
            proj, x = kept["proj"][i], kept["x"][i + 1]
            gate = proj[:, self.memory.columns:]
            d_proj, dz, d_before = torch.empty_like(proj), torch.empty_like(x), torch.empty_like(x)
            binding.bagel_block_join_grad(kept["z"][i], x, dx, dy, gate=gate, act="silu", post_weight=v[f"post{i}"], scale=v[f"scale{i}"],
                                          pre_weight=v[f"pre{i + 1}"], eps=EPS, d_branch=dz, d_gate=d_proj[:, self.memory.columns:], d_resid=d_before,
                                          d_post_weight=grads[f"post{i}"], d_scale=grads[f"scale{i}"], d_pre_weight=grads[f"pre{i + 1}"])
            dx = d_before
            grads[f"out{i}"] = dz.t() @ kept["h"][i]
            self.memory.backward(proj, v, i, kept["offsets"], kept["initial"][i] if kept["initial"] else None, kept["memory"][i], dz @ w[f"out{i}"], d_proj, grads)
            grads[f"in{i}"] = d_proj.t() @ kept["y"][i]
            dy = d_proj @ w[f"in{i}"]
        d_x0 = torch.empty_like(kept["x"][0])
        binding.bagel_block_join_grad(None, kept["x"][0], dx, dy, pre_weight=v["pre0"], eps=EPS, d_resid=d_x0, d_pre_weight=grads["pre0"])
        grads["obs"] = d_x0.t() @ kept["obs"]
        return grads

    def update(self, grads: Dict[str, torch.Tensor], lr: float = 1e-3, weight_decay: float = 0.01, grad_scale: Optional[torch.Tensor] = None,
               max_norm: Optional[float] = None):
        """One step of AdamW: the matrices with weight decay and their working copies, the vectors without.  max_norm: the gradients of all are clipped to that
        norm together, which is returned (a tensor); where it is not finite, nothing changes."""
        self.updates += 1
        norm = None
        if max_norm is not None:
            norm, factor = (torch.empty(1, device="cuda") for _ in range(2))
            binding.bagel_clip_norm(list(grads.values()), max_norm, norm, factor, grad_scale=grad_scale)
            grad_scale = factor
        groups = ((self.matrices, weight_decay, [self.work[k] for k in self.matrices]), (self.vectors, 0.0, None))
        for i, (group, decay, copy) in enumerate(groups):
            moments = [self.moments[k] for k in group]
            binding.bagel_adamw_step(list(group.values()), [grads[k] for k in group], [s.m for s in moments], [s.v for s in moments], self.updates,
                                     m_scale=[s.m_scale for s in moments], v_scale=[s.v_scale for s in moments], copy=copy, lr=lr,
                                     weight_decay=decay, grad_scale=grad_scale, run=len(groups) * self.seed + i)
        return norm

    # ------------------------------------------------------------------------------------------------ one control period at a time
    def start(self, machines: int) -> List[torch.Tensor]:
        """The memory of so many machines, empty."""
        return [self.memory.start(machines) for _ in range(self.blocks)]

    def step(self, observations: torch.Tensor, memory: List[torch.Tensor]) -> torch.Tensor:
        """Actions for one observation of every machine; the memory goes on by one step in place."""
        v, w = self.vectors, self.work
        x = observations.to(self.dtype) @ w["obs"].t()
        y = torch.empty_like(x)
        binding.bagel_block_join(None, x, None, y, pre_weight=v["pre0"], eps=EPS)
        for i in range(self.blocks):
            proj = y @ w[f"in{i}"].t()
            h = self.memory.step(proj, v, i, memory[i])
            binding.bagel_block_join(h @ w[f"out{i}"].t(), x, x, y, gate=proj[:, self.memory.columns:], act="silu", post_weight=v[f"post{i}"],
                                     scale=v[f"scale{i}"], pre_weight=v[f"pre{i + 1}"], eps=EPS)
        return y @ w["act"].t()


class _Channels:
    """A number for every channel: the gated recurrence."""

    def __init__(self, width: int):
        self.width, self.columns = width, 2 * width

    def vectors(self, i: int):
        # memories of a few steps up to a few hundred
        return {f"bias{i}": torch.linspace(0.0, 5.0, self.width, device="cuda")}

    def _parts(self, proj):
        return proj[:, :self.width], proj[:, self.width:2 * self.width]

    def forward(self, proj, v, i, offsets, initial):
        h = torch.empty(proj.shape[0], self.width, dtype=proj.dtype, device="cuda")
        carry = torch.empty(binding.bagel_recurrence_carry_rows(proj.shape[0]), self.width, device="cuda")
        binding.bagel_recurrence(*self._parts(proj), h, offsets, bias=v[f"bias{i}"], initial=initial, carry=carry)
        return h, carry

    def backward(self, proj, v, i, offsets, initial, carry, dh, d_proj, grads):
        binding.bagel_recurrence_grad(*self._parts(proj), dh, *self._parts(d_proj), offsets, carry, bias=v[f"bias{i}"], initial=initial, d_bias=grads[f"bias{i}"])

    def start(self, machines: int):
        return torch.zeros(machines, self.width, device="cuda")

    def step(self, proj, v, i, memory):
        h = torch.empty(proj.shape[0], self.width, dtype=proj.dtype, device="cuda")
        binding.bagel_recurrence_step(*self._parts(proj), memory, h, bias=v[f"bias{i}"])
        return h


class _Heads:
    """A matrix for every head: linear attention, and the layer norm of every head of its results."""

    def __init__(self, width: int, heads: int):
        self.width, self.heads, self.columns = width, heads, 3 * width
        self.scale = (width // heads) ** -0.5
        # memories of a few steps up to a few hundred
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2.0, 8.0, heads, device="cuda")))

    def vectors(self, i: int):
        return {f"norm{i}": torch.ones(self.width, device="cuda"), f"shift{i}": torch.zeros(self.width, device="cuda")}

    def _parts(self, proj):
        return [proj[:, k * self.width:(k + 1) * self.width].unflatten(1, (self.heads, -1)) for k in range(3)]

    def _normed(self, o, v, i):
        h = torch.empty_like(o)
        binding.bagel_layer_norm(o, h, weight=v[f"norm{i}"], bias=v[f"shift{i}"], groups=self.heads, eps=EPS)
        return h

    def forward(self, proj, v, i, offsets, initial):
        o = torch.empty(proj.shape[0], self.width, dtype=proj.dtype, device="cuda")
        binding.bagel_linear_attention(*self._parts(proj), o.unflatten(1, (self.heads, -1)), offsets, self.log_decay, scale=self.scale, initial=initial)
        return self._normed(o, v, i), o

    def backward(self, proj, v, i, offsets, initial, o, dh, d_proj, grads):
        d_o = torch.empty_like(o)
        binding.bagel_layer_norm_grad(o, dh, d_o, weight=v[f"norm{i}"], groups=self.heads, eps=EPS, d_weight=grads[f"norm{i}"], d_bias=grads[f"shift{i}"])
        binding.bagel_linear_attention_grad(*self._parts(proj), d_o.unflatten(1, (self.heads, -1)), *self._parts(d_proj), offsets, self.log_decay, scale=self.scale,
                                            initial=initial)

    def start(self, machines: int):
        return torch.zeros(machines, self.heads, self.width // self.heads, self.width // self.heads, device="cuda")

    def step(self, proj, v, i, memory):
        o = torch.empty(proj.shape[0], self.width, dtype=proj.dtype, device="cuda")
        binding.bagel_linear_attention_step(*self._parts(proj), memory, o.unflatten(1, (self.heads, -1)), self.log_decay, scale=self.scale)
        return self._normed(o, v, i)


class _Moments:
    def __init__(self, p: torch.Tensor, bits: int):
        kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
        self.m, self.v = (torch.zeros(p.shape, device=p.device).to(kind) for _ in range(2))
        blocks = -(-p.numel() // binding.ADAMW_BLOCK)
        self.m_scale, self.v_scale = (torch.zeros(blocks, device=p.device) if bits == 8 else None for _ in range(2))


def recorded_rollouts(name: str = "tiny", trial: int = 0):
    """States[B, H+1, d_s] and goals[B, H, d_g] of the configuration's rollouts, and the actions[B, H, d_a] of its memoryless policy."""
    from . import synth
    cfg = synth.CONFIGS[name]
    inp = {k: torch.from_numpy(a).cuda() for k, a in synth.make_inputs(cfg, trial=trial).items()}
    ctx = binding.Bagel(binding.dims_from_config(cfg))
    ctx.bagel_prepare_samples(*(inp[k] for k in ("X", "y", "lengthscale", "signal_var", "noise_var", "omega", "phase", "w", "eps")))
    states, loss = torch.empty(cfg.H + 1, cfg.B, cfg.d_s, device="cuda"), torch.empty(1, device="cuda")
    ctx.bagel_rollout_loss(inp["theta"], inp["s0"], inp["goals"], loss, states=states)
    torch.cuda.synchronize()
    ctx.close()
    a, at = torch.cat([states[:-1], inp["goals"]], 2), 0
    for i, (rows, columns) in enumerate(cfg.layer_shapes):
        weights, bias = inp["theta"][at:at + rows * columns].view(rows, columns), inp["theta"][at + rows * columns:at + rows * columns + rows]
        at += rows * columns + rows
        a = a @ weights.t() + bias
        if i + 1 < len(cfg.layer_shapes):
            a = torch.tanh(a)
    if cfg.act_bound > 0:
        a = cfg.act_bound * torch.tanh(a)
    return states.transpose(0, 1).contiguous(), inp["goals"].transpose(0, 1).contiguous(), a.transpose(0, 1).contiguous()


def imitate(policy: MemoryPolicy, observations: torch.Tensor, actions: torch.Tensor, updates: int, lr: float = 3e-3,
            max_norm: Optional[float] = None) -> List[float]:
    """Trains on whole trajectories, observations[B, H, d_in] and actions[B, H, d_out], by the mean squared error; the losses."""
    trajectories = observations.shape[0]
    obs, want = observations.flatten(0, 1), actions.flatten(0, 1)
    losses = []
    for _ in range(updates):
        got, kept = policy.forward(obs, trajectories)
        off = got.float() - want
        losses.append(off.square().mean())
        policy.update(policy.backward(kept, off * (2.0 / off.numel())), lr=lr, max_norm=max_norm)
    return torch.stack(losses).tolist()


def main():
    states, goals, actions = recorded_rollouts()
    actions = (actions - actions.mean()) / actions.std()
    seen = torch.cat([states[:, :-1, :1], goals], 2)                 # a position and its goal, no velocity
    for bits, heads in ((32, 0), (8, 0), (32, 4)):
        policy = MemoryPolicy(seen.shape[2], actions.shape[2], width=128, blocks=2, state_bits=bits, heads=heads)
        losses = imitate(policy, seen, actions, 300, max_norm=1.0 if heads else None)
        whole = policy.forward(seen.flatten(0, 1), seen.shape[0])[0].float().view(actions.shape)
        memory = policy.start(seen.shape[0])
        steps = torch.stack([policy.step(seen[:, t], memory) for t in range(seen.shape[1])], 1).float()
        print(f"{f'{heads} heads' if heads else 'channels'}, moments in {bits} bits: mean squared error {losses[0]:.4f} -> {losses[-1]:.5f} of a variance of 1, whole trajectories and single "
              f"steps differ by {float((whole - steps).norm() / whole.norm()):.1e}")


if __name__ == "__main__":
    main()
