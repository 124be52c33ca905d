"""The policy whose memory is a matrix for every head: attention, norm of the heads, join, clipping and update put together, against torch's automatic
differentiation of the same policy in 64 bits."""
import pytest
import torch

from paper_2202_13638_amd import binding, memory_policy as mp

pytestmark = pytest.mark.gpu


def _reference(policy, observations, lengths, parameters):
    """Actions of the policy in 64 bits, step by step."""
    p, heads = parameters, policy.memory.heads
    decay = torch.exp(policy.memory.log_decay.double().cpu())[:, None, None]

    def norm(z, weight):
        return z / torch.sqrt(z.square().mean(-1, keepdim=True) + mp.EPS) * weight

    out, at, d = [], 0, policy.width
    for n in lengths:
        x = observations[at:at + n] @ p["obs"].t()
        at += n
        y = norm(x, p["pre0"])
        for i in range(policy.blocks):
            q, k, v, gate = (y @ p[f"in{i}"].t()).split(d, 1)
            q, k, v = (t.view(n, heads, -1) for t in (q, k, v))
            S, rows = torch.zeros(heads, d // heads, d // heads, dtype=torch.float64), []
            for t in range(n):
                S = decay * S + k[t, :, :, None] * v[t, :, None, :]
                rows.append(policy.memory.scale * torch.matmul(q[t][:, None], S)[:, 0])
            o = torch.stack(rows)
            c = o - o.mean(2, keepdim=True)
            h = (c / torch.sqrt(c.square().mean(2, keepdim=True) + mp.EPS)).view(n, d) * p[f"norm{i}"] + p[f"shift{i}"]
            z = h @ p[f"out{i}"].t()
            x = x + p[f"scale{i}"] * gate * torch.sigmoid(gate) * norm(z, p[f"post{i}"])
            y = norm(x, p[f"pre{i + 1}"])
        out.append(y @ p["act"].t())
    return torch.cat(out)


def test_gradient_of_the_whole_policy_with_heads():
    """In 32 bits: some dozen operators one after the other, each within 1e-5 of its own; a first row's answer of a head is q.k v, whose norm brings out what is small
    beside its deviation, so held to 1e-3 of a parameter's gradient."""
    lengths = [150, 1, 37]
    policy = mp.MemoryPolicy(3, 2, width=24, blocks=2, dtype=torch.float32, heads=3)
    g = torch.Generator().manual_seed(1)
    obs, weights = torch.randn(188, 3, generator=g), torch.randn(188, 2, generator=g)
    offsets = torch.tensor([0, 150, 151, 188], dtype=torch.int32).cuda()
    got, kept = policy.forward(obs.cuda(), offsets)
    grads = policy.backward(kept, weights.cuda())
    parameters = {k: t.double().cpu().requires_grad_() for k, t in {**policy.matrices, **policy.vectors}.items()}
    want = _reference(policy, obs.double(), lengths, parameters)
    off = got.double().cpu() - want.detach()
    assert float(off.norm() / want.detach().norm()) < 1e-3
    (want * weights.double()).sum().backward()
    for k, p in parameters.items():
        assert float((grads[k].double().cpu() - p.grad).norm() / p.grad.norm()) < 1e-3, k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_updates_are_clipped_by_the_norm_of_all_gradients(dtype):
    policies = [mp.MemoryPolicy(3, 2, width=32, blocks=1, dtype=dtype, heads=2) for _ in range(2)]
    obs = torch.randn(100, 3, generator=torch.Generator().manual_seed(2)).cuda()
    got, kept = policies[0].forward(obs, 4)
    grads = policies[0].backward(kept, torch.ones_like(got))
    want = torch.sqrt(sum(t.double().square().sum() for t in grads.values()))
    norm = policies[0].update(grads, max_norm=0.5)
    assert abs(float(norm) - float(want)) <= 1e-6 * float(want)
    # the same update by the factor itself
    factor = (0.5 / (want + 1e-6)).clamp(max=1.0).float().reshape(1)
    policies[1].update(grads, grad_scale=factor)
    for k, p in policies[0].matrices.items():
        off = (p - policies[1].matrices[k]).abs().max()
        assert float(off) <= 1e-7 * float(p.abs().max()) + 1e-8, k       # factors a rounding apart, updates of 1e-3
    # what is not finite changes nothing
    before = {k: p.clone() for k, p in policies[0].matrices.items()}
    grads["act"].view(-1)[0] = float("inf")
    norm = policies[0].update(grads, max_norm=0.5)
    assert not torch.isfinite(norm).any() and all(torch.equal(p, before[k]) for k, p in policies[0].matrices.items())


def test_a_policy_with_heads_trains_and_steps():
    states, goals, actions = mp.recorded_rollouts()
    actions = (actions - actions.mean()) / actions.std()
    seen = torch.cat([states[:, :-1, :1], goals], 2)
    policy = mp.MemoryPolicy(seen.shape[2], 1, width=64, blocks=2, heads=4)
    losses = mp.imitate(policy, seen, actions, 20, max_norm=1.0)
    assert all(x == x and x < float("inf") for x in losses)
    # a step at a time it acts as it does over whole trajectories: in 32 bits, as sums of rows and sums along them are rounded differently
    policy = mp.MemoryPolicy(seen.shape[2], 1, width=64, blocks=2, heads=4, dtype=torch.float32)
    whole = policy.forward(seen.flatten(0, 1), seen.shape[0])[0].view(actions.shape)
    memory = policy.start(seen.shape[0])
    steps = torch.stack([policy.step(seen[:, t], memory) for t in range(seen.shape[1])], 1)
    assert float((whole - steps).norm() / whole.norm()) < 1e-3


def test_heads_must_divide_the_width():
    with pytest.raises(ValueError, match="heads"):
        mp.MemoryPolicy(3, 2, width=32, blocks=1, heads=5)
    assert binding.ATTENTION_MAX_WIDTH >= 32
