"""Calls of the policy with memory that other tests do not make."""
import pytest
import torch

from paper_2202_13638_amd import binding, memory_policy as mp


@pytest.mark.parametrize("width,heads", [(32, 5), (32, -4), (32, 64), (256, 1), (3 * 129, 3)])
def test_heads_that_the_attention_does_not_take_are_refused(width, heads):
    with pytest.raises(ValueError, match="heads must divide the width"):
        mp.MemoryPolicy(3, 2, width=width, blocks=1, heads=heads)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,max_norm", [(2, 1e-3), (2, None), (0, 1e-3)])
def test_imitation_makes_the_updates_of_its_gradients(heads, max_norm):
    """Its parameters are those of AdamW for the gradients of the mean squared error, times the factor that brings their norm down: computed here in 64 bits."""
    policies = [mp.MemoryPolicy(3, 2, width=32, blocks=1, dtype=torch.float32, heads=heads) for _ in range(2)]
    g = torch.Generator().manual_seed(3)
    seen, actions = torch.randn(6, 40, 3, generator=g).cuda(), torch.randn(6, 40, 2, generator=g).cuda()
    loss, = mp.imitate(policies[0], seen, actions, 1, lr=1e-2, max_norm=max_norm)
    p = policies[1]
    got, kept = p.forward(seen.flatten(0, 1), 6)
    off = got - actions.flatten(0, 1)
    assert abs(loss - float(off.double().square().mean())) <= 1e-6 * loss
    grads = p.backward(kept, off * (2.0 / off.numel()))
    norm = torch.sqrt(sum(x.double().square().sum() for x in grads.values()))
    factor = 1.0 if max_norm is None else min(1.0, max_norm / (float(norm) + 1e-6))
    assert max_norm is None or factor < 0.5
    for k, before in {**p.matrices, **p.vectors}.items():
        x = grads[k].double() * factor
        # the first step: m / (1 - beta1) = x, v / (1 - beta2) = x^2, and a weight decay of 0.01 for matrices
        want = before.double() * (1 - (1e-2 * 0.01 if k in p.matrices else 0.0)) - 1e-2 * x / (x.abs() + 1e-8)
        after = {**policies[0].matrices, **policies[0].vectors}[k]
        # 32 bits round the parameter three times: 1 - lr weight_decay (of almost one), its product with the parameter, and what the step makes of that, each by 2^-24 of the
        # parameter or of it and the step; and what the step of 1e-2 is made of some ten times
        assert float((after.double() - want).abs().max()) <= 3 * 2.0 ** -24 * (float(before.abs().max()) + 1e-2) + 10 * 2.0 ** -24 * 1e-2, k
        assert not torch.equal(after, before), k
