"""Calls of linear attention, layer norm and clipping that their documentation allows: sizes, places and values that other tests do not have."""
import ctypes as C
import itertools
import random

import pytest
import torch

from paper_2202_13638_amd import binding
from test_more_operators import (HALF_ULP, TYPES, _attention_all, _attention_check, _attention_inputs, _attention_struct, _attention_want, _near)

gpu = pytest.mark.gpu


# segments are a number of chunks of rows that depends on the type: of eight and of four chunks, 16 bits keep what 32 bits make odd
@pytest.mark.parametrize("heads,states", [(8, 8), (16, 8), (4, 1), (8, 2), (1, 1)])
def test_work_spaces_are_for_every_type(heads, states):
    """What bagel_linear_attention_workspace says without a type is enough for each.  (The calls are refused, for the place of the work space, before anything is launched.)"""
    for rows, sequences, grad in itertools.product(list(range(1000, 70000, 1777)) + [15000, 30000, 31000, 32000], [1, 2, 50], [False, True]):
        size = binding.bagel_linear_attention_workspace(rows, sequences, heads, states, 64, 64, grad)
        for dtype, offsets in itertools.product([0, 1, 2], [None, 0x10000]):
            if offsets is None and rows % sequences:
                continue
            a = _attention_struct(rows=rows, sequences=sequences, heads=heads, states=states, key_width=64, value_width=64, dtype=dtype, offsets=offsets,
                                  workspace=0x10004, workspace_bytes=size)
            for k in ("query", "key", "value", "out", "d_out", "d_query", "d_key", "d_value"):
                setattr(a, k + "_head", 64)
                setattr(a, k + "_stride", 64 * heads)
            lib = binding.load()
            assert (lib.bagel_linear_attention_grad if grad else lib.bagel_linear_attention)(C.byref(a), None) == binding.EINVAL
            assert b"16 bytes" in lib.bagel_last_error(None), (rows, sequences, dtype, offsets, lib.bagel_last_error(None))


@gpu
@pytest.mark.parametrize("dk,dv,heads,states,offsets", [(8, 8, 1, 1, False), (8, 8, 2, 1, True), (8, 72, 1, 1, True), (2, 3, 1, 1, True)])
def test_more_memories_than_a_grid_has_workgroups_for(dk, dv, heads, states, offsets):
    """A grid has fewer than 2^32 threads: with workgroups of 256 (512 for values wider than 64), sequences of one row and an empty one at the end."""
    n, t = (1 << (23 if dv > 64 else 24)) + 5, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(1)

    def whole(*shape):
        return torch.randint(-4, 5, shape, generator=g, device="cuda", dtype=torch.int8).to(t)

    q, k, v, d = whole(n, heads, dk), whole(n, states, dk), whole(n, states, dv), whole(n, heads, dv)
    at = n
    if offsets:                                      # two rows behind the last sequence, whose results are zero
        at = torch.arange(n, device="cuda", dtype=torch.int32).clamp(max=n - 2)
    ld = torch.tensor([-0.5], device="cuda")
    out, dq, dk_, dv_ = (torch.full_like(x, 7.0) for x in (d, q, k, v))
    binding.bagel_linear_attention(q, k, v, out, at, ld)
    binding.bagel_linear_attention_grad(q, k, v, d, dq, dk_, dv_, at, ld)
    last = n - 2 if offsets else n
    for a in range(0, n, 1 << 22):                   # whole numbers, which 32 bits hold
        b = min(a + (1 << 22), n)
        x, y, z, e = (i[a:b].float() for i in (q, k, v, d))
        qk, de = (x * y).sum(2, keepdim=True), (e * z).sum(2, keepdim=True)
        for got, want in ((out, qk * z), (dq, de * y), (dk_, (de * x).sum(1, keepdim=True)), (dv_, (qk * e).sum(1, keepdim=True))):
            want[max(last - a, 0):] = 0
            assert torch.equal(got[a:b], want.to(t)), a


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", [[150, 0, 3], [700]], ids=["chunks", "shared out"])
@pytest.mark.parametrize("heads,states,dk,dv", [(2, 2, 64, 64), (8, 2, 64, 40), (4, 2, 128, 128), (2, 2, 5, 3)])
def test_a_decay_that_is_nan_is_seen(heads, states, dk, dv, lengths, dtype):
    """In what it multiplies, and in nothing of the other memory: whole sequences, gradients and steps alike."""
    t = TYPES[dtype]
    x, _ = _attention_inputs(lengths, heads, states, dk, dv, t, seed=4)
    ld = torch.tensor([-0.1, float("nan")])
    want, _ = _attention_want(x, lengths, ld, 0.2)
    _, terms = _attention_want(x, lengths, torch.full_like(ld, -0.1), 0.2)
    got = _attention_all(x, lengths, ld, 0.2)
    for k, g in got.items():
        g, w = g.cpu(), want[k]
        assert torch.equal(g.isnan(), w.isnan()), k
        _near(torch.where(w.isnan(), torch.zeros_like(g), g), torch.nan_to_num(w), k, terms[k], 0.0 if dtype == "f32" else 2 * HALF_ULP[t])
    state, out = x["initial"].cuda(), torch.zeros(len(lengths), heads, dv, dtype=t, device="cuda")
    q, k, v = (x[i][:len(lengths)].cuda() for i in "qkv")
    if len(q) == len(lengths):
        binding.bagel_linear_attention_step(q, k, v, state, out, ld.cuda())
        assert state[:, 1].isnan().all() and out[:, heads // 2:].isnan().all() and state[:, 0].isfinite().all() and out[:, :heads // 2].isfinite().all()


def test_tensors_of_heads_that_meet():
    """Against sets of places: refused only where an entry is shared, and always where rows and heads are the same distances apart."""
    from paper_2202_13638_amd import _marshal
    g, buffer, hits, misses = random.Random(1), torch.zeros(400), 0, 0
    place = torch.arange(400.0)

    def refused(x, y):
        try:
            _marshal.apart(("x",), (x,), ("y",), (y,))
        except ValueError as e:
            assert str(e) == "x may not be in the place of y"
            return True
        return False

    for _ in range(20000):
        rows = g.randint(1, 5)
        strides = [(g.choice([0, 3, 7, 12, 24, 40]), g.choice([0, 2, 5, 8, 13]))] * 2
        if g.random() < 0.2:
            strides[1] = (g.randint(0, 40), g.randint(0, 13))
        shapes = [(rows, g.randint(1, 4), g.randint(1, 6)) for _ in range(2)]
        x, y = (torch.as_strided(buffer, s, (*d, 1), g.randint(0, 60)) for s, d in zip(shapes, strides))
        a, b = (set(torch.as_strided(place, t.shape, t.stride(), t.storage_offset()).flatten().tolist()) for t in (x, y))
        if a & b:
            hits += refused(x, y)
            assert refused(x, y) or strides[0] != strides[1], (x.shape, x.stride(), x.storage_offset(), y.shape, y.stride(), y.storage_offset())
        else:
            misses += 1
            assert not refused(x, y)
    assert hits > 3000 and misses > 3000
    # and results with each other
    x = torch.zeros(6, 2, 8)
    with pytest.raises(ValueError, match="a may not be in the place of b"):
        _marshal.apart(("a", "b"), (x, x), (), ())
    _marshal.apart(("a", "b"), (x, None), ("c",), (None,))


@gpu
def test_results_in_the_place_of_what_is_read_are_refused():
    """The gradients of keys read the values again where both are not made at once, and rows with what is not finite are gone through once more."""
    proj = torch.randn(90, 3 * 2 * 16, device="cuda", dtype=torch.bfloat16)
    q, k, v = (proj[:, 32 * i:32 * i + 32].unflatten(1, (2, 16)) for i in range(3))
    d, ld, new = torch.randn(90, 2, 16, device="cuda", dtype=torch.bfloat16), torch.tensor([-0.1, -0.2], device="cuda"), torch.empty_like(proj).unflatten(1, (3, 2, 16))
    for out in (q, k, v, proj[:, 8:40].unflatten(1, (2, 16))):
        with pytest.raises(ValueError, match="out may not be in the place of"):
            binding.bagel_linear_attention(q, k, v, out, 1, ld)
        with pytest.raises(ValueError, match="out may not be in the place of"):
            binding.bagel_linear_attention_step(q, k, v, torch.zeros(90, 2, 16, 16, device="cuda"), out, ld)
    for place, bad in itertools.product(range(3), (q, k, v, d)):
        outs = [new[:, i] for i in range(3)]
        outs[place] = bad
        with pytest.raises(ValueError, match=f"d_{('query', 'key', 'value')[place]} may not be in the place of"):
            binding.bagel_linear_attention_grad(q, k, v, d, *outs, 1, ld)
    with pytest.raises(ValueError, match="d_query may not be in the place of d_value"):
        binding.bagel_linear_attention_grad(q, k, v, d, new[:, 0], new[:, 1], new[:, 0], 1, ld)
    # parts of one projection, and of the gradient of one, lie apart
    out = torch.empty_like(d)
    binding.bagel_linear_attention(q, k, v, out, 1, ld)
    binding.bagel_linear_attention_grad(q, k, v, d, new[:, 0], new[:, 1], new[:, 2], 1, ld)
    wide = torch.zeros(90, 4 * 2 * 16, device="cuda", dtype=torch.bfloat16)              # and a result beside what is read
    wide[:, :96] = proj
    parts = [wide[:, 32 * i:32 * i + 32].unflatten(1, (2, 16)) for i in range(4)]
    binding.bagel_linear_attention(*parts, 1, ld)
    assert torch.equal(parts[3], out) and torch.equal(wide[:, :96], proj)


@gpu
def test_the_norm_has_a_place_of_its_own():
    """The factor is written behind it; the factor itself may take the place of the scale that it is made of."""
    g, one, other = [torch.full((5000,), 2.0, device="cuda")], torch.full((1,), 0.5, device="cuda"), torch.zeros(1, device="cuda")
    with pytest.raises(ValueError, match="norm may not be in the place of"):
        binding.bagel_clip_norm(g, 1.0, other, other)
    with pytest.raises(ValueError, match="norm may not be in the place of"):
        binding.bagel_clip_norm(g, 1.0, one, other, grad_scale=one)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    binding.bagel_clip_norm(g, 1.0, norm, factor, grad_scale=one)
    binding.bagel_clip_norm(g, 1.0, other, one, grad_scale=one)
    assert torch.equal(one, factor) and torch.equal(other, norm) and abs(float(norm) - 5000 ** 0.5) < 1e-4


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,heads,states,dk,dv", [([700], 8, 2, 64, 64), ([700], 4, 1, 128, 128), ([40, 2900], 8, 1, 24, 16), ([90, 1500], 2, 2, 64, 64)],
                         ids=["joined by the parts", "wide", "joined by a launch", "a head to a memory"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_in_a_sequence_that_is_shared_out(bad, lengths, heads, states, dk, dv, dtype):
    """Segments before it, and the rows of its own segment before it, have the results that they have without it; those behind it have nothing finite where it is."""
    t, n = TYPES[dtype], sum(lengths)
    at, first = n - 333, n - lengths[-1]
    x, _ = _attention_inputs(lengths, heads, states, dk, dv, t, seed=51)
    ld = torch.full((states,), -0.004)
    want, terms = _attention_want(x, lengths, ld, 0.2)
    clean = _attention_all(x, lengths, ld, 0.2)
    g = heads // states
    before, behind = slice(0, at), slice(at + 1, n)
    for name, places in (("v", {"out": before}), ("k", {"out": before, "d_query": before}), ("q", {"d_key": behind, "d_value": behind}), ("d_out", {"d_key": behind, "d_value": behind})):
        y = dict(x, **{name: x[name].clone()})
        y[name][at, 0, 2] = bad
        got = _attention_all(y, lengths, ld, 0.2)
        for k, rows in places.items():
            _near(got[k][rows], want[k][rows], f"{k} for {name}", terms[k][rows], 0.0 if dtype == "f32" else 2 * HALF_ULP[t])
        for k, v in got.items():                     # the other sequence and the other memory
            if k in ("final", "d_initial"):
                assert torch.equal(v[:-1], clean[k][:-1]) and torch.equal(v[:, 1:], clean[k][:, 1:]), (name, k)
            else:
                of = g if v.shape[1] == heads else 1
                assert torch.equal(v[:first], clean[k][:first]) and torch.equal(v[:, of:], clean[k][:, of:]), (name, k)
        hit = {"v": got["out"][at:, :g, 2], "k": got["out"][at:, :g], "q": got["d_value"][first:at + 1, 0], "d_out": got["d_value"][first:at + 1, 0, 2]}[name]
        assert not hit.isfinite().any(), name
        if name in "vk":
            assert not got["final"][-1, 0].isfinite().all()
        else:
            assert not got["d_initial"][-1, 0].isfinite().all()


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1600, 1536, 1537])
def test_segments_of_four_chunks(rows, dtype):
    """Many memories of one sequence, so that segments are longer than the least: of an even number of chunks."""
    t = TYPES[dtype]
    x, ld = _attention_inputs([rows], 256, 64, 8, 12, t, seed=52)
    ld = torch.linspace(-0.05, -0.001, 64)
    want, terms = _attention_want(x, [rows], ld, 0.2)
    _attention_check(_attention_all(x, [rows], ld, 0.2), want, terms, t)
