"""How many bits linear attention keeps of what it works with, in 16-bit types.

Of whole numbers nothing is rounded but the results: with no decay and a scale that is a power of two, the products of a chunk's rows, the memories and all sums are whole
numbers (times that power) below 2^24, which 32 bits hold, and what becomes an operand is below 2^16, which a sum of two bfloat16 numbers holds (2^22 of
float16).  So every result is the definition's, rounded once, to the bit."""
import pytest
import torch

from test_more_operators import HALF_ULP, TYPES, _attention_all, _attention_inputs, _attention_want

gpu = pytest.mark.gpu
SIZES = [(2, 2, 64, 64), (8, 2, 64, 64), (4, 2, 128, 128), (2, 2, 128, 128), (8, 2, 24, 100), (8, 2, 100, 24)]


def _whole(shape, seed, most, t=torch.float32):
    return torch.randint(-most, most + 1, shape, generator=torch.Generator().manual_seed(seed)).to(t)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,states,dk,dv", SIZES)
@pytest.mark.parametrize("lengths", [[64], [150, 0, 3], [400, 30]], ids=["a chunk", "chunks", "shared out"])
def test_nothing_but_the_results_is_rounded(lengths, heads, states, dk, dv, dtype):
    t, rows, n = TYPES[dtype], sum(lengths), len(lengths)
    # a memory is at most 500 + 4 x 4 x 400 x 4 heads < 2^16, a result at most 4 x 128 times that < 2^24
    x = dict(q=_whole((rows, heads, dk), 1, 4, t), k=_whole((rows, states, dk), 2, 4, t), v=_whole((rows, states, dv), 3, 4, t), d_out=_whole((rows, heads, dv), 4, 4, t),
             initial=_whole((n, states, dk, dv), 5, 500), d_final=_whole((n, states, dk, dv), 6, 500) * 2.0 ** -6)
    ld, scale = torch.zeros(states), 2.0 ** -6
    want, _ = _attention_want(x, lengths, ld, scale)
    got = _attention_all(x, lengths, ld, scale)
    for k, g in got.items():
        w = want[k].float()
        assert torch.equal(w.double(), want[k]), k                   # (32 bits hold it)
        assert torch.equal(g.cpu(), w.to(g.dtype)), f"{k}: {int((g.cpu() != w.to(g.dtype)).sum())} of {g.numel()} differ"


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,states,dk,dv", SIZES)
def test_results_are_as_near_as_their_type_allows(heads, states, dk, dv, dtype):
    """With decays.  A result y = x + e before its rounding is at most |round(x) - x| + 2 |e| from x, as round(y) is no farther from y than round(x) is.  e: terms with an
    operand in two parts are off by u^2 of themselves, u half a unit of the type, with signs of their own, as the terms have; a hundred sums in 32 bits make 2^-24 each, below 2^-20
    together.  Held to twice what that makes of the norm."""
    t, u = TYPES[dtype], HALF_ULP[TYPES[dtype]]
    x, ld = _attention_inputs([300, 70], heads, states, dk, dv, t, seed=3)
    want, _ = _attention_want(x, [300, 70], ld, dk ** -0.5)
    got = _attention_all(x, [300, 70], ld, dk ** -0.5)
    for k in ("out", "d_query", "d_key", "d_value"):
        rounding = float((want[k].to(t).double() - want[k]).norm() / want[k].norm())
        off = float((got[k].double().cpu() - want[k]).norm() / want[k].norm())
        assert off <= rounding + 4 * (u * u + 2.0 ** -20), (k, off, rounding)
