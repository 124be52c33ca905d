"""The policy with memory: the library's operators put together, against torch's automatic differentiation of the same policy in 64 bits."""
import pytest
import torch

from paper_2202_13638_amd import memory_policy as mp

pytestmark = pytest.mark.gpu


def _reference(policy, observations, lengths, parameters):
    """Actions of the policy in 64 bits, step by step."""
    p = parameters

    def norm(z, weight):
        return z / torch.sqrt(z.square().mean(-1, keepdim=True) + mp.EPS) * weight

    out, at, d = [], 0, policy.width
    for n in lengths:
        x = observations[at:at + n] @ p["obs"].t()
        at += n
        y = norm(x, p["pre0"])
        for i in range(policy.blocks):
            value, forget, gate = (y @ p[f"in{i}"].t()).split(d, 1)
            q, h, rows = torch.sigmoid(-(forget + p[f"bias{i}"])), torch.zeros(d, dtype=torch.float64), []
            for t in range(n):
                h = h + q[t] * (value[t] - h)
                rows.append(h)
            z = torch.stack(rows) @ p[f"out{i}"].t()
            x = x + p[f"scale{i}"] * gate * torch.sigmoid(gate) * norm(z, p[f"post{i}"])
            y = norm(x, p[f"pre{i + 1}"])
        out.append(y @ p["act"].t())
    return torch.cat(out)


def test_gradient_of_the_whole_policy():
    """In 32 bits: some ten operators one after the other, each within 1e-5 of its own; held to 1e-4 of a parameter's gradient."""
    lengths = [150, 1, 37]
    policy = mp.MemoryPolicy(3, 2, width=24, blocks=2, dtype=torch.float32)
    g = torch.Generator().manual_seed(1)
    obs, weights = torch.randn(188, 3, generator=g), torch.randn(188, 2, generator=g)
    offsets = torch.tensor([0, 150, 151, 188], dtype=torch.int32).cuda()
    got, kept = policy.forward(obs.cuda(), offsets)
    grads = policy.backward(kept, weights.cuda())
    parameters = {k: t.double().cpu().requires_grad_() for k, t in {**policy.matrices, **policy.vectors}.items()}
    want = _reference(policy, obs.double(), lengths, parameters)
    off = got.double().cpu() - want.detach()
    assert float(off.norm() / want.detach().norm()) < 1e-4
    (want * weights.double()).sum().backward()
    for k, p in parameters.items():
        assert float((grads[k].double().cpu() - p.grad).norm() / p.grad.norm()) < 1e-4, k


@pytest.mark.parametrize("bits", [32, 8])
def test_it_learns_to_act_from_positions_alone(bits):
    states, goals, actions = mp.recorded_rollouts()
    actions = (actions - actions.mean()) / actions.std()
    seen = torch.cat([states[:, :-1, :1], goals], 2)
    policy = mp.MemoryPolicy(seen.shape[2], 1, width=64, blocks=2, state_bits=bits)
    losses = mp.imitate(policy, seen, actions, 150)
    assert losses[-1] < 0.1 * losses[0] and losses[-1] < 0.1          # the variance of what it learns is 1
    # a step at a time it acts as it does over whole trajectories: activations in bf16, a few roundings of 2^-8 apart
    whole = policy.forward(seen.flatten(0, 1), seen.shape[0])[0].float().view(actions.shape)
    memory = policy.start(seen.shape[0])
    steps = torch.stack([policy.step(seen[:, t], memory) for t in range(seen.shape[1])], 1).float()
    assert float((whole - steps).norm() / whole.norm()) < 0.05
