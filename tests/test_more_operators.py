"""Layer norm, linear attention with a decay for every head and clipping by the norm of all gradients against plain implementations in 64 bits.

Tolerances.  u is half a unit in the last place: 2^-24, 2^-8 or 2^-11 of a value in 32 bits, bfloat16 and float16.  A result is rounded once, u of itself.  Before that
stand sums and products in 32 bits, together below 1e-5 of the sum of the magnitudes that a result is made of (a few dozen roundings of 2^-24 in
a row, and an exponential whose argument carries a few more).  Linear attention also rounds what is multiplied to the type of its operands: the weights of a chunk's
rows and the memory before a chunk, u each of what they are (none in 32 bits).  So an entry of a result is off by at most u |result| + (2 u + 1e-5) of the
sum of magnitudes, and, as roundings of inputs with random signs do not add up but their squares do (u^2 / 3 each for three of them), the
whole result by u of its norm: held to 1.5 u, and 1e-5 in 32 bits."""
import ctypes as C
import math

import pytest
import torch

from paper_2202_13638_amd import binding

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
WORK = 1e-5
NAN = float("nan")


def _normal(shape, seed, dtype=torch.float32, scale=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + mean).to(dtype)


def _near(got, want, name, terms, operands=0.0):
    """`terms`: the sums of the magnitudes that the entries are made of; `operands`: what rounding operands may take of them."""
    assert got.shape == want.shape, name
    if want.numel() == 0:
        return
    g, w = got.double().cpu(), want.double().cpu()
    bound = HALF_ULP[got.dtype] * w.abs() * 1.01 + (WORK + operands) * terms.double().cpu()
    if got.dtype == torch.float16:
        bound = bound + 2.0 ** -25                   # its smallest numbers are this far apart, twice
    off = (g - w).abs()
    inside = bool((off <= bound).all())
    assert inside, f"{name}: off by {float(off.max()):.3g}, at most {float((off - bound).max()):.3g} too much"


# -------------------------------------------------------------------------------------------------------------- layer norm
def _parts(x, groups):
    return x.reshape(x.shape[0], groups, -1)


def _norm_ref(x, weight, bias, groups, eps):
    c = _parts(x.double(), groups)
    c = c - c.mean(2, keepdim=True)
    n = (c / torch.sqrt(c.square().mean(2, keepdim=True) + eps)).reshape(x.shape)
    w = torch.ones(x.shape[1], dtype=torch.float64) if weight is None else weight.double()
    out = n * w + (0 if bias is None else bias.double())
    # a mean is a sum of a part's entries, so its error is relative to the largest of them, over the deviation
    reach = _parts(x.double().abs(), groups).amax(2, keepdim=True) / torch.sqrt(c.square().mean(2, keepdim=True) + eps)
    terms = (n.abs() + reach.expand(-1, -1, c.shape[2]).reshape(x.shape)) * w.abs() + (0 if bias is None else bias.double().abs())
    return out, terms


def _norm_grad_ref(x, d, weight, groups, eps):
    c = _parts(x.double(), groups)
    c = c - c.mean(2, keepdim=True)
    r = 1 / torch.sqrt(c.square().mean(2, keepdim=True) + eps)
    n = c * r
    w = torch.ones(x.shape[1], dtype=torch.float64) if weight is None else weight.double()
    e = _parts(d.double() * w, groups)
    dx = r * (e - e.mean(2, keepdim=True) - n * (e * n).mean(2, keepdim=True))
    reach = 1 + _parts(x.double().abs(), groups).amax(2, keepdim=True) * r           # what an error of the mean is of n
    terms = r * reach * (e.abs() + e.abs().mean(2, keepdim=True) + (n.abs() + reach) * (e * n).abs().mean(2, keepdim=True))
    n, reach = n.reshape(x.shape), reach.expand_as(e).reshape(x.shape)
    dd = d.double()
    return ({"d_x": dx.reshape(x.shape), "d_weight": (dd * n).sum(0), "d_bias": dd.sum(0)},
            {"d_x": terms.reshape(x.shape), "d_weight": (dd.abs() * (n.abs() + reach)).sum(0), "d_bias": dd.abs().sum(0)})


def _norm_case(x, d, weight, bias, groups, eps=1e-5, view=lambda t: t.cuda()):
    g = [t if t is None else t.cuda() for t in (weight, bias)]
    gx, gd = view(x), view(d)
    out, d_x = view(torch.full_like(x, NAN)), view(torch.full_like(x, NAN))
    binding.bagel_layer_norm(gx, out, weight=g[0], bias=g[1], groups=groups, eps=eps)
    want, terms = _norm_ref(x, weight, bias, groups, eps)
    _near(out, want, "out", terms)
    dw, db = (torch.full((x.shape[1],), NAN, device="cuda") for _ in range(2))
    binding.bagel_layer_norm_grad(gx, gd, d_x, weight=g[0], groups=groups, eps=eps, d_weight=dw, d_bias=db)
    want, terms = _norm_grad_ref(x, d, weight, groups, eps)
    for name, got in (("d_x", d_x), ("d_weight", dw), ("d_bias", db)):
        _near(got, want[name], name, terms[name])
    return out, d_x, dw, db


NORM_SIZES = [(1, 1, 1), (3, 2, 1), (2, 63, 1), (5, 64, 1), (4, 65, 1), (7, 255, 1), (9, 256, 1), (3, 777, 1), (33, 1000, 1), (2, 1026, 1), (5, 2048, 1),
              (3, 2056, 1), (2, 4096, 1), (3, 5001, 1), (2, 8192, 1), (2, 16384, 1), (1, 16383, 1), (7, 12, 12), (19, 24, 8), (50, 512, 8),
              (33, 1024, 16), (21, 17 * 40, 17), (40, 3 * 333, 3), (5, 2 * 8000, 2), (9, 100 * 3, 100), (6, 24 * 130, 24)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,groups", NORM_SIZES)
def test_layer_norm_and_its_gradient(rows, width, groups, dtype):
    t = TYPES[dtype]
    k = rows + width
    _norm_case(_normal((rows, width), k, t, 2.0, 0.5), _normal((rows, width), k + 1, t), _normal((width,), k + 2, scale=0.2, mean=1.0),
               _normal((width,), k + 3, scale=0.3), groups)


@gpu
@pytest.mark.parametrize("rows,width,groups,dtype", [(70001, 40, 1, "f32"), (20003, 64, 2, "bf16"), (9000, 6 * 24, 6, "f16"), (4001, 17 * 8, 17, "bf16"),
                                                     (3000, 23 * 136, 23, "bf16"), (2000, 1040, 1, "f32"), (1500, 7 * 700, 7, "f16"), (1100, 4100, 1, "bf16"),
                                                     (900, 1000, 500, "f32")])
def test_layer_norm_of_more_rows_than_there_are_places(rows, width, groups, dtype):
    t = TYPES[dtype]
    x, d = _normal((rows, width), 1, t, 2.0, 0.5), _normal((rows, width), 2, t)
    weight, bias = _normal((width,), 3, scale=0.2, mean=1.0), _normal((width,), 4, scale=0.3)
    first = _norm_case(x, d, weight, bias, groups)
    again = _norm_case(x, d, weight, bias, groups)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,stride,width,groups", [(0, 640, 512, 1), (8, 1040, 512, 8), (1, 515, 512, 4), (3, 131, 64, 1), (0, 200, 77, 7), (2, 2050, 2048, 1)])
def test_layer_norm_of_strided_rows(start, stride, width, groups, dtype):
    t, rows = TYPES[dtype], 13

    def view(x):
        buffer = torch.full((start + rows * stride,), 7.0, dtype=t, device="cuda")
        buffers.append(buffer)
        v = buffer[start:].as_strided((rows, width), (stride, 1), start)
        v.copy_(x)
        return v

    buffers = []
    _norm_case(_normal((rows, width), 1, t, 2.0, 0.5), _normal((rows, width), 2, t), None, None, groups, view=view)
    for b in buffers:                                # nothing is written between the rows
        keep = torch.ones_like(b, dtype=torch.bool)
        keep[start:].as_strided((rows, width), (stride, 1), start).fill_(False)
        assert bool((b[keep] == 7.0).all())


@gpu
def test_layer_norm_in_place_and_parts_left_out():
    x, d = (_normal((50, 300), k, torch.bfloat16).cuda() for k in (1, 2))
    weight = _normal((300,), 3, mean=1.0).cuda()
    out, d_x = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    binding.bagel_layer_norm(x, out, weight=weight)
    binding.bagel_layer_norm_grad(x, d, d_x, weight=weight, d_weight=dw, d_bias=db)
    y = x.clone()
    binding.bagel_layer_norm(y, y, weight=weight)
    assert torch.equal(y, out)
    for into in ("x", "d"):
        a, b = x.clone(), d.clone()
        binding.bagel_layer_norm_grad(a, b, a if into == "x" else b, weight=weight)
        assert torch.equal(a if into == "x" else b, d_x)
    for left in ("d_weight", "d_bias"):
        got = {k: torch.full((300,), NAN, device="cuda") for k in ("d_weight", "d_bias") if k != left}
        binding.bagel_layer_norm_grad(x, d, weight=weight, **got)
        assert all(torch.equal(v, {"d_weight": dw, "d_bias": db}[k]) for k, v in got.items())
    # no rows: no gradient
    binding.bagel_layer_norm(x[:0], out[:0])
    binding.bagel_layer_norm_grad(x[:0], d[:0], d_weight=dw, d_bias=db)
    assert not dw.any() and not db.any()


@gpu
def test_layer_norm_of_constant_rows_and_large_means():
    # a row of one value has no deviation: its norm is the bias, to eps; a large mean is taken off before anything is squared
    x = torch.cat([torch.full((1, 512), 3.0), torch.full((1, 512), -1000.0), _normal((2, 512), 1, mean=1000.0), torch.zeros(1, 512)])
    bias = _normal((512,), 2)
    _norm_case(x, _normal(x.shape, 3), None, bias, 1)
    _norm_case(x, _normal(x.shape, 3), None, bias, 4)


@gpu
def test_a_nan_stays_in_its_part():
    for bad in (NAN, float("inf")):
        x = _normal((6, 256), 1)
        x[2, 70] = bad
        out, d_x = torch.empty(6, 256, device="cuda"), torch.empty(6, 256, device="cuda")
        binding.bagel_layer_norm(x.cuda(), out, groups=4)
        binding.bagel_layer_norm_grad(x.cuda(), torch.ones(6, 256, device="cuda"), d_x, groups=4)
        for t in (out, d_x):
            hit = t.isnan().cpu()
            want = torch.zeros(6, 256, dtype=torch.bool)
            want[2, 64:128] = True
            assert torch.equal(hit, want)


# -------------------------------------------------------------------------------------------------------- linear attention
def _attention_ref(q, k, v, initial, lengths, log_decay, scale):
    """out and final, row after row, by the definition; differentiable."""
    rows, heads, _ = q.shape
    states, group = k.shape[1], heads // k.shape[1]
    decay, at, out, final = torch.exp(log_decay)[:, None, None], 0, [], []
    for i, n in enumerate(lengths):
        S = initial[i]
        for t in range(at, at + n):
            S = decay * S + k[t, :, :, None] * v[t, :, None, :]
            out.append(scale * torch.matmul(q[t].view(states, group, -1), S).reshape(heads, -1))
        at += n
        final.append(S)
    out = torch.stack(out) if out else q.new_zeros(0, heads, v.shape[2])
    pad = rows - at
    return torch.cat([out, out.new_zeros(pad, *out.shape[1:])]), torch.stack(final)


def _attention_inputs(lengths, heads, states, dk, dv, t, seed=0, behind=0):
    rows, k = sum(lengths) + behind, 10 * seed
    x = dict(q=_normal((rows, heads, dk), k + 1, t), k=_normal((rows, states, dk), k + 2, t), v=_normal((rows, states, dv), k + 3, t),
             initial=_normal((len(lengths), states, dk, dv), k + 4), d_out=_normal((rows, heads, dv), k + 5, t),
             d_final=_normal((len(lengths), states, dk, dv), k + 6))
    return x, torch.linspace(-1.0, -0.004, states) if states > 1 else torch.tensor([-0.02])


def _offsets(lengths):
    return torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)), dtype=torch.int32).cuda()


def _attention_all(x, lengths, ld, scale, offsets=None, cuda=lambda d: {k: t.cuda() for k, t in d.items()}):
    """Results of the calls, in memory that held NaN."""
    g = cuda(x)
    like = lambda t: torch.full(t.shape, NAN, dtype=t.dtype, device="cuda")
    r = dict(out=like(x["d_out"]), final=like(x["initial"]), d_query=like(x["q"]), d_key=like(x["k"]), d_value=like(x["v"]), d_initial=like(x["initial"]))
    at = _offsets(lengths) if offsets is None else offsets
    binding.bagel_linear_attention(g["q"], g["k"], g["v"], r["out"], at, ld.cuda(), scale=scale, initial=g["initial"], final=r["final"])
    binding.bagel_linear_attention_grad(g["q"], g["k"], g["v"], g["d_out"], r["d_query"], r["d_key"], r["d_value"], at, ld.cuda(), scale=scale,
                                        initial=g["initial"], d_final=g["d_final"], d_initial=r["d_initial"])
    return r


def _attention_want(x, lengths, ld, scale):
    """Results in 64 bits, and the sums of the magnitudes that they are made of."""
    def results(x):
        leaves = [x[k].double().requires_grad_() for k in ("q", "k", "v", "initial")]
        out, final = _attention_ref(*leaves, lengths, ld.double(), scale)
        loss = (out * x["d_out"].double()).sum() + (final * x["d_final"].double()).sum()
        d = torch.autograd.grad(loss, leaves) if loss.requires_grad else [torch.zeros_like(t) for t in leaves]
        return dict(out=out.detach(), final=final.detach(), d_query=d[0], d_key=d[1], d_value=d[2], d_initial=d[3])
    return results(x), results({k: t.abs() for k, t in x.items()})


def _attention_check(got, want, terms, t):
    for name in got:
        operands = 2 * HALF_ULP[t] if t != torch.float32 and got[name].dtype == t else 0.0
        _near(got[name], want[name], name, terms[name], operands)
        w = want[name].double()
        if w.numel() >= 64 and float(w.norm()) > 0:
            off = float((got[name].double().cpu() - w).norm() / w.norm())
            assert off < max(1e-5, 1.5 * HALF_ULP[got[name].dtype]), f"{name}: off by {off:.3g} of its norm"


LENGTHS = [[1], [5, 0, 0, 3], [64], [63, 1, 65], [129, 7, 0, 200, 1], [300], [1] * 40]
WIDTHS = [(2, 1, 64, 64), (3, 3, 40, 77), (4, 2, 128, 128), (1, 1, 1, 1), (8, 2, 65, 8), (2, 2, 16, 128), (6, 2, 127, 33)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,states,dk,dv", WIDTHS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: "x".join(map(str, v[:6])))
def test_linear_attention_and_its_gradient(lengths, heads, states, dk, dv, dtype):
    t = TYPES[dtype]
    x, ld = _attention_inputs(lengths, heads, states, dk, dv, t, seed=dk + len(lengths))
    scale = dk ** -0.5
    want, terms = _attention_want(x, lengths, ld, scale)
    _attention_check(_attention_all(x, lengths, ld, scale), want, terms, t)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_attention_along_a_long_sequence(dtype):
    """Long enough to be shared out along its rows; two sequences of another length behind it.  The same bits every time."""
    t, lengths = TYPES[dtype], [2500, 3, 700]
    x, ld = _attention_inputs(lengths, 2, 1, 64, 48, t, seed=3)
    ld = torch.tensor([-0.002])
    want, terms = _attention_want(x, lengths, ld, 0.125)
    got = _attention_all(x, lengths, ld, 0.125)
    _attention_check(got, want, terms, t)
    again = _attention_all(x, lengths, ld, 0.125)
    assert all(torch.equal(got[k], again[k]) for k in got)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ld", [-math.inf, 0.0, -30.0, -1e-6])
def test_linear_attention_of_extreme_decays(ld, dtype):
    t, lengths = TYPES[dtype], [150, 0, 20]
    x, _ = _attention_inputs(lengths, 2, 2, 32, 32, t, seed=5)
    decays = torch.tensor([ld, -0.1])
    want, terms = _attention_want(x, lengths, decays, 0.2)
    _attention_check(_attention_all(x, lengths, decays, 0.2), want, terms, t)


@gpu
@pytest.mark.parametrize("tail", [1, 64, 200])
def test_linear_attention_rows_behind_the_last_sequence(tail):
    """What they hold, NaN here, is not used, and their results are zero."""
    t, lengths = torch.bfloat16, [70, 0, 33]
    x, ld = _attention_inputs(lengths, 4, 2, 64, 40, t, seed=7, behind=tail)
    want, terms = _attention_want({k: v[:103] if v.shape[0] > 103 else v for k, v in x.items()}, lengths, ld, 0.125)
    for k in ("q", "k", "v", "d_out"):
        x[k][103:] = NAN
    got = _attention_all(x, lengths, ld, 0.125)
    for k in ("out", "d_query", "d_key", "d_value"):
        assert not got[k][103:].any()
        got[k] = got[k][:103]
    _attention_check(got, want, terms, t)


@gpu
@pytest.mark.parametrize("bad", [NAN, math.inf])
def test_linear_attention_keeps_what_is_not_finite_in_its_sequence_and_memory(bad):
    lengths = [70, 90, 10]
    x, ld = _attention_inputs(lengths, 4, 2, 64, 64, torch.bfloat16, seed=8)
    clean = _attention_all(x, lengths, ld, 0.125)
    x["v"][100, 1, 3] = bad
    got = _attention_all(x, lengths, ld, 0.125)
    for k in got:
        a, b = got[k].cpu(), clean[k].cpu()
        if k in ("final", "d_initial"):
            assert torch.equal(a[[0, 2]], b[[0, 2]]) and torch.equal(a[1, 0], b[1, 0])
        else:
            heads = slice(0, 2) if a.shape[1] == 4 else slice(0, 1)
            assert torch.equal(a[:70], b[:70]) and torch.equal(a[160:], b[160:]) and torch.equal(a[:, heads], b[:, heads])
    assert not got["out"][100, 2:, 3].isfinite().any() and not got["final"][1, 1, :, 3].isfinite().all()


@gpu
def test_linear_attention_equal_lengths_without_offsets():
    x, ld = _attention_inputs([90] * 5, 4, 2, 64, 64, torch.bfloat16, seed=9)
    a, b = _attention_all(x, [90] * 5, ld, 0.125), _attention_all(x, [90] * 5, ld, 0.125, offsets=5)
    assert all(torch.equal(a[k], b[k]) for k in a)


@gpu
def test_linear_attention_parts_left_out():
    """Without initial and d_final they are zero; results that are not wanted are not needed."""
    lengths = [70, 0, 140]
    x, ld = _attention_inputs(lengths, 4, 2, 64, 40, torch.float32, seed=10)
    x["initial"].zero_()
    x["d_final"].zero_()
    want = _attention_all(x, lengths, ld, 0.3)
    g, at, ld = {k: t.cuda() for k, t in x.items()}, _offsets(lengths), ld.cuda()
    out = torch.empty_like(g["d_out"])
    binding.bagel_linear_attention(g["q"], g["k"], g["v"], out, at, ld, scale=0.3)
    assert torch.equal(out, want["out"])
    for name, place in (("d_query", 0), ("d_key", 1), ("d_value", 2), ("d_initial", 3)):
        got = torch.full_like(want[name], NAN)
        outs = [got if place == k else None for k in range(3)]
        binding.bagel_linear_attention_grad(g["q"], g["k"], g["v"], g["d_out"], *outs, at, ld, scale=0.3, d_initial=got if place == 3 else None)
        assert torch.equal(got, want[name]), name


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["parts of a projection", "heads before rows", "odd start", "broadcast"])
def test_linear_attention_of_strided_heads(layout, dtype):
    t, lengths = TYPES[dtype], [100, 41]
    x, ld = _attention_inputs(lengths, 4, 2, 40, 33, t, seed=11)
    if layout == "broadcast":                        # one key for all memories, one value for all rows
        x["k"][:] = x["k"][:, :1]
        x["v"][:] = x["v"][:1]
    want, terms = _attention_want(x, lengths, ld, 0.2)
    views = []

    def cuda(d):
        r = {k: v.cuda() for k, v in d.items()}
        if layout == "parts of a projection":
            proj = torch.cat([r[k].flatten(1) for k in "qkv"], 1)
            r["q"], r["k"], r["v"] = proj[:, :160].view(-1, 4, 40), proj[:, 160:240].view(-1, 2, 40), proj[:, 240:].view(-1, 2, 33)
        elif layout == "heads before rows":
            for k in ("q", "k", "v", "d_out"):
                r[k] = r[k].transpose(0, 1).contiguous().transpose(0, 1)
        elif layout == "odd start":
            for k in ("q", "k", "v", "d_out"):
                r[k] = torch.cat([r[k].new_zeros(3), r[k].flatten()])[3:].view(r[k].shape)
        else:
            r["k"], r["v"] = r["k"][:, :1].expand(-1, 2, -1), r["v"][:1].expand(141, -1, -1)
        views.append(r)
        return r

    _attention_check(_attention_all(x, lengths, ld, 0.2, cuda=cuda), want, terms, t)
    # and results in strided places: nothing is written between them
    r = views[0]
    for name, like, place in (("d_query", "q", 0), ("d_key", "k", 1), ("d_value", "v", 2)):
        rows, heads, width = x[like].shape
        buffer = torch.full((rows, heads + 1, width + 5), 7.0, dtype=t, device="cuda")
        outs = [buffer[:, :heads, 1:width + 1] if place == k else None for k in range(3)]
        binding.bagel_linear_attention_grad(r["q"], r["k"], r["v"], r["d_out"], *outs, _offsets(lengths), ld.cuda(), scale=0.2, initial=r["initial"],
                                            d_final=r["d_final"])
        _attention_check({name: outs[place].contiguous()}, want, terms, t)
        buffer[:, :heads, 1:width + 1] = 7.0
        assert bool((buffer == 7.0).all()), name


@gpu
def test_linear_attention_of_one_memory_for_many_heads_of_far_rows():
    """Places beyond 2^31 entries."""
    t, rows = torch.bfloat16, 130
    big = torch.zeros(rows * (1 << 25), dtype=t, device="cuda")
    x, ld = _attention_inputs([rows], 2, 1, 32, 24, t, seed=12)
    want, terms = _attention_want(x, [rows], ld, 0.2)

    def cuda(d):
        r = {k: v.cuda() for k, v in d.items()}
        for n, k in enumerate(("q", "k", "v", "d_out")):
            heads, width = d[k].shape[1:]
            far = big.as_strided(d[k].shape, (1 << 25, width, 1), n * 1024)
            far.copy_(r[k])
            r[k] = far
        return r

    _attention_check(_attention_all(x, [rows], ld, 0.2, cuda=cuda), want, terms, t)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,heads,states,dk,dv", [(1, 1, 1, 1, 1), (1, 8, 8, 64, 64), (5, 4, 2, 128, 128), (3, 6, 3, 40, 77), (200, 8, 1, 64, 32),
                                                     (9, 2, 2, 127, 128), (0, 2, 1, 8, 8), (2, 64, 4, 16, 16), (3000, 2, 2, 33, 20)])
def test_linear_attention_step(rows, heads, states, dk, dv, dtype):
    t = TYPES[dtype]
    x, ld = _attention_inputs([1] * rows, heads, states, dk, dv, t, seed=13)
    g = {k: v.cuda() for k, v in x.items()}
    out, state = torch.full((rows, heads, dv), NAN, dtype=t, device="cuda"), g["initial"].clone()
    binding.bagel_linear_attention_step(g["q"], g["k"], g["v"], state, out, ld.cuda(), scale=0.3)
    if rows == 0:
        return
    S = torch.exp(ld.double())[:, None, None] * x["initial"].double() + x["k"].double()[..., None] * x["v"].double()[..., None, :]
    A = torch.exp(ld.double())[:, None, None] * x["initial"].double().abs() + x["k"].double().abs()[..., None] * x["v"].double().abs()[..., None, :]
    q = x["q"].double().view(rows, states, heads // states, dk)
    _near(state, S, "state", A)
    _near(out, 0.3 * torch.matmul(q, S).view(out.shape), "out", 0.3 * torch.matmul(q.abs(), A).view(out.shape))


@gpu
def test_linear_attention_step_is_the_sequence_one_row_at_a_time():
    """In 32 bits, steps and whole sequences differ by their sums' order only."""
    machines, n = 3, 80
    x, ld = _attention_inputs([n] * machines, 4, 2, 64, 64, torch.float32, seed=14)
    want, terms = _attention_want(x, [n] * machines, ld, 0.125)
    g = {k: v.cuda() for k, v in x.items()}
    q, k, v = (g[i].view(machines, n, *g[i].shape[1:]) for i in "qkv")
    state, outs = g["initial"].clone(), []
    for i in range(n):
        out = torch.empty(machines, 4, 64, device="cuda")
        binding.bagel_linear_attention_step(q[:, i], k[:, i], v[:, i], state, out, ld.cuda(), scale=0.125)
        outs.append(out)
    _near(torch.stack(outs, 1).view(-1, 4, 64), want["out"], "out", terms["out"])
    _near(state, want["final"], "state", terms["final"])


@gpu
def test_more_gradients_against_differences():
    """Central differences of the calls themselves, in 32 bits: their results are exact to 1e-6 of some dozens here, so a difference over 2^-4 to 1e-3."""
    step, lengths = 2.0 ** -5, [70, 20]
    x, ld = _attention_inputs(lengths, 2, 1, 24, 20, torch.float32, seed=15)
    grads = _attention_all(x, lengths, ld, 0.2)

    def loss(y):
        r = _attention_all(y, lengths, ld, 0.2)
        return float((r["out"].double().cpu() * x["d_out"].double()).sum() + (r["final"].double().cpu() * x["d_final"].double()).sum())

    # linear in each input, so a central difference has no error of its own
    for name, grad in (("q", "d_query"), ("k", "d_key"), ("v", "d_value"), ("initial", "d_initial")):
        way = _normal(x[name].shape, 16)
        up, down = (loss({**x, name: x[name] + s * step * way}) for s in (1, -1))
        want = float((grads[grad].double().cpu() * way.double()).sum())
        assert abs((up - down) / (2 * step) - want) < 1e-3 * float(grads[grad].double().norm()), name

    a, d, w, b = _normal((40, 96), 1), _normal((40, 96), 2), _normal((96,), 3, mean=1.0), _normal((96,), 4)
    dx, dw, db = torch.empty(40, 96, device="cuda"), torch.empty(96, device="cuda"), torch.empty(96, device="cuda")
    binding.bagel_layer_norm_grad(a.cuda(), d.cuda(), dx, weight=w.cuda(), groups=3, d_weight=dw, d_bias=db)

    def norm_loss(a, w, b):
        out = torch.empty(40, 96, device="cuda")
        binding.bagel_layer_norm(a.cuda(), out, weight=w.cuda(), bias=b.cuda(), groups=3)
        return float((out.double().cpu() * d.double()).sum())

    # x: the third derivative of the norm over step^2 / 6 is below 1e-3 of the gradient for steps of 2^-8 of its deviation
    for k, grad, size in ((0, dx, 2.0 ** -8), (1, dw, step), (2, db, step)):
        inputs = [a, w, b]
        way = _normal(inputs[k].shape, 17)
        up, down = (norm_loss(*[t + s * size * way if i == k else t for i, t in enumerate(inputs)]) for s in (1, -1))
        want = float((grad.double().cpu() * way.double()).sum())
        assert abs((up - down) / (2 * size) - want) < 2e-3 * float(grad.double().norm()), k


# ---------------------------------------------------------------------------------------------------------------- clipping
def _clip_case(shapes, t, max_norm, grad_scale=0.37, scale=1e-2, write="all", shift=0):
    """t: the tensors' type, or types that they have in turn."""
    types = t if isinstance(t, list) else [t]
    g = [_normal(s, 20 + i, types[i % len(types)], scale) for i, s in enumerate(shapes)]

    def placed(x):
        return torch.cat([x.new_zeros(shift), x.flatten()]).cuda()[shift:].view(x.shape)

    gg = [placed(x) for x in g]
    outs = None if write == "none" else [placed(torch.full_like(x, 7.0)) if write == "all" or i % 2 else None for i, x in enumerate(g)]
    norm, factor = torch.full((1,), NAN, device="cuda"), torch.full((1,), NAN, device="cuda")
    scale = None if grad_scale is None else torch.tensor([grad_scale], device="cuda")
    binding.bagel_clip_norm(gg, max_norm, norm, factor, grad_scale=scale, out=outs)
    s = 1.0 if grad_scale is None else float(torch.tensor(grad_scale))
    want = math.sqrt(sum(float(x.double().square().sum()) for x in g)) * abs(s)
    f = s * min(1.0, max_norm / (want + 1e-6))
    # the norm is rounded once, the factor is made of it by four operations
    assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.01 and abs(float(factor) - f) <= 6 * 2.0 ** -24 * abs(f)
    for x, o in zip(g, outs or []):
        if o is not None:
            _near(o, x.double() * f, "out", (x.double() * f).abs())
    assert all(torch.equal(a.cpu(), b) for a, b in zip(gg, g))
    return norm, factor


CLIP_SHAPES = [(256, 5), (256,), (256, 256), (1,), (777, 333), (2,), (8193,), (0,), (16384,)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_norm", [1.0, 0.01, math.inf, 0.0])
@pytest.mark.parametrize("write", ["none", "all", "some"])
def test_clip_norm(write, max_norm, dtype):
    _clip_case(CLIP_SHAPES, TYPES[dtype], max_norm, write=write)
    _clip_case([(3,)], TYPES[dtype], max_norm, grad_scale=None, write=write)


@gpu
@pytest.mark.parametrize("write", ["none", "all"])
def test_clip_norm_of_several_types(write):
    types = [torch.bfloat16, torch.float32, torch.float16]
    _clip_case(CLIP_SHAPES, types, 0.5, write=write)
    _clip_case([(40,), (7,), (9,), (300,)], types, 0.5, write=write)
    _clip_case([(20000,)] * 150, types, 0.5, write=write)


@gpu
@pytest.mark.parametrize("shift", [1, 2, 3, 5])
@pytest.mark.parametrize("dtype", TYPES)
def test_clip_norm_at_odd_starts(shift, dtype):
    _clip_case([(300, 7), (9000,), (1,), (5,)], TYPES[dtype], 0.5, grad_scale=-2.0, shift=shift)


@gpu
@pytest.mark.parametrize("count,first,second", [(95, 5, 20000), (96, 300, 7), (97, 7, 70000), (300, 10000, 33), (1000, 3, 3)])
def test_clip_norm_of_many_tensors(count, first, second):
    """More than a launch takes, with few workgroups before many and many before few."""
    shapes = [(first if i < count // 2 else second,) for i in range(count)]
    a = _clip_case(shapes, torch.bfloat16, 0.3)
    b = _clip_case(shapes, torch.bfloat16, 0.3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@gpu
def test_clip_norm_of_large_and_small_values():
    # squares that 32 bits do not hold
    _clip_case([(5000,), (70000,)], torch.float32, 1.0, grad_scale=1e-10, scale=1e30)
    _clip_case([(5000,), (70000,)], torch.float32, 1.0, grad_scale=None, scale=1e-30)
    _clip_case([(100,)], torch.bfloat16, 1.0, grad_scale=1e-10, scale=1e30)


@gpu
def test_clip_norm_of_nothing_of_zeros_and_of_what_is_not_finite():
    norm, factor = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    binding.bagel_clip_norm([], 1.0, norm, factor)
    assert float(norm) == 0.0 and float(factor) == 1.0
    binding.bagel_clip_norm([torch.zeros(50, device="cuda"), torch.zeros(0, device="cuda")], 1.0, norm, factor)
    assert float(norm) == 0.0 and float(factor) == 1.0
    for bad in (NAN, math.inf, -math.inf):
        g = [_normal((9000,), 1).cuda(), _normal((40,), 2).cuda()]
        g[1][3] = bad
        kept, out = [t.clone() for t in g], [torch.full_like(t, 7.0) for t in g]
        binding.bagel_clip_norm(g, 1.0, norm, factor, out=out)
        assert not norm.isfinite() and factor.isnan() and all(bool((t == 7.0).all()) for t in out)
        binding.bagel_clip_norm(g, 1.0, norm, factor, out=g)
        assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(g, kept))
        # and the update leaves everything as it was
        p, m, v = torch.ones(9000, device="cuda"), torch.zeros(9000, device="cuda"), torch.zeros(9000, device="cuda")
        binding.bagel_adamw_step([p], g[:1], [m], [v], 1, grad_scale=factor)
        assert bool((p == 1).all()) and not m.any()
    scale = torch.tensor([math.inf], device="cuda")
    binding.bagel_clip_norm([torch.ones(5, device="cuda")], 1.0, norm, factor, grad_scale=scale)
    assert factor.isnan()


@gpu
def test_clip_norm_in_place_is_clip_norm_and_repeats():
    g = [_normal((3000,), 1, torch.bfloat16).cuda(), _normal((17, 5), 2, torch.bfloat16).cuda()]
    out = [torch.empty_like(t) for t in g]
    norm, factor = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    binding.bagel_clip_norm(g, 1.0, norm, factor, out=out)
    binding.bagel_clip_norm(g, 1.0, norm, factor, out=g)
    assert all(torch.equal(a, b) for a, b in zip(g, out))
    binding.bagel_clip_norm(g, 1.0, norm, factor)
    assert abs(float(norm) - 1.0) < 2.0 ** -8                 # entries were rounded by half a unit at most


# --------------------------------------------------------------------------------------------- streams, graphs, together
def _all_calls(stream=None):
    """A training step's calls in a row, of fixed tensors: launch(), outputs, inputs."""
    t, lengths, h, n, dk, dv = torch.bfloat16, [300, 0, 77, 500], 4, 2, 64, 48
    x, ld = _attention_inputs(lengths, h, n, dk, dv, t, seed=30)
    x = {k: v.cuda() for k, v in x.items()}
    rows, at, ld = 877, _offsets(lengths), ld.cuda()
    weight, bias = _normal((h * dv,), 31, mean=1.0).cuda(), _normal((h * dv,), 32).cuda()
    new = lambda *s, dtype=t: torch.zeros(s, dtype=dtype, device="cuda")
    f = torch.float32
    out, normed, d_o, final, d_initial = new(rows, h, dv), new(rows, h * dv), new(rows, h * dv), new(4, n, dk, dv, dtype=f), new(4, n, dk, dv, dtype=f)
    dq, dk_, dv_, dw, db = new(rows, h, dk), new(rows, n, dk), new(rows, n, dv), new(h * dv, dtype=f), new(h * dv, dtype=f)
    norm, factor, clipped = new(1, dtype=f), new(1, dtype=f), [new(rows, h, dk), new(rows, n, dk), new(rows, n, dv)]
    state, step_out = x["initial"][:, :, :, :].clone(), new(4, h, dv)
    grad_space = torch.empty(max(16, binding.bagel_linear_attention_workspace(rows, 4, h, n, dk, dv, True)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def launch():
        k = dict(stream=stream)
        binding.bagel_linear_attention(x["q"], x["k"], x["v"], out, at, ld, scale=0.125, initial=x["initial"], final=final, **k)
        binding.bagel_layer_norm(out.view(rows, -1), normed, weight=weight, bias=bias, groups=h, **k)
        binding.bagel_layer_norm_grad(out.view(rows, -1), x["d_out"].view(rows, -1), d_o, weight=weight, groups=h, d_weight=dw, d_bias=db, **k)
        binding.bagel_linear_attention_grad(x["q"], x["k"], x["v"], d_o.view(rows, h, dv), dq, dk_, dv_, at, ld, scale=0.125, initial=x["initial"],
                                            d_final=x["d_final"], d_initial=d_initial, workspace=grad_space, **k)
        binding.bagel_clip_norm([dq, dk_, dv_], 1.0, norm, factor, out=clipped, **k)
        binding.bagel_linear_attention_step(x["q"][:4], x["k"][:4], x["v"][:4], state, step_out, ld, **k)

    return launch, [out, normed, d_o, final, d_initial, dq, dk_, dv_, dw, db, norm, factor, *clipped, state, step_out], x


@gpu
def test_more_operators_on_another_stream():
    launch, want, _ = _all_calls()
    launch()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    launch, got, _ = _all_calls(side)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        launch()
    side.synchronize()
    for a, b in zip(want[:-2], got[:-2]):
        assert torch.equal(a, b)


@gpu
def test_more_operators_in_a_graph():
    """Replayed with new inputs, eager work and synchronisations in between; every replay is the eager result."""
    launch, got, x = _all_calls()
    eager, want, y = _all_calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    before = [t.clone() for t in got]
    with torch.cuda.stream(side):
        launch()
    torch.cuda.current_stream().wait_stream(side)
    for t, b in zip(got, before):
        t.copy_(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        launch()
    for k in range(4):
        for name in ("q", "k", "v", "d_out"):
            new = _normal(x[name].shape, 100 * k + len(name), torch.bfloat16).cuda()
            x[name].copy_(new)
            y[name].copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        eager()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), k


# --------------------------------------------------------------------------------------------------------------- refusals
def _refused(call, args, text, *more):
    lib = binding.load()
    assert getattr(lib, call)(*more, C.byref(args), None) == binding.EINVAL
    message = lib.bagel_last_error(None).decode()
    assert message.startswith(call + ":") and text in message, message


def _norm_struct(**kw):
    a = binding._Norm()
    a.rows, a.width, a.dtype, a.groups, a.eps = 4, 32, 0, 2, 1e-5
    for k in ("x", "out", "d_out", "d_x"):
        setattr(a, k, 0x10000)
        setattr(a, k + "_stride", 32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("call", ["bagel_layer_norm", "bagel_layer_norm_grad"])
@pytest.mark.parametrize("change,text", [
    (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(width=16385), "width"), (dict(dtype=3), "dtype"), (dict(groups=0), "groups"),
    (dict(groups=3), "groups"), (dict(eps=0.0), "eps"), (dict(eps=NAN), "eps"), (dict(x=None), "x is needed"), (dict(x_stride=31), "stride"),
    (dict(x=0x10002), "stride")])
def test_layer_norm_refuses(call, change, text):
    _refused(call, _norm_struct(**change), text)


@pytest.mark.parametrize("change,text", [
    (dict(d_out=None), "d_out"), (dict(d_weight=0x10000), "workspace"), (dict(d_bias=0x10000, workspace=0x10000, workspace_bytes=16), "too small"),
    (dict(d_weight=0x10000, workspace=0x10008, workspace_bytes=1 << 20), "16 bytes"), (dict(d_x_stride=4), "stride")])
def test_layer_norm_grad_refuses(change, text):
    _refused("bagel_layer_norm_grad", _norm_struct(**change), text)
    _refused("bagel_layer_norm", _norm_struct(out=None), "out")


def _attention_struct(**kw):
    a = binding._Attention()
    a.rows, a.key_width, a.value_width, a.heads, a.states, a.dtype, a.sequences, a.scale = 6, 32, 16, 4, 2, 1, 2, 1.0
    a.log_decay = a.workspace = a.state = 0x10000
    a.workspace_bytes = 1 << 24
    for k in ("query", "key", "value", "out", "d_out", "d_query", "d_key", "d_value"):
        setattr(a, k, 0x10000)
        setattr(a, k + "_head", 32)
        setattr(a, k + "_stride", 128)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("call", ["bagel_linear_attention", "bagel_linear_attention_grad"])
@pytest.mark.parametrize("change,text", [
    (dict(rows=-1), "rows"), (dict(rows=1 << 28), "rows"), (dict(key_width=0), "key_width"), (dict(value_width=129), "value_width"),
    (dict(heads=0), "heads"), (dict(states=0), "states"), (dict(states=3), "divide"), (dict(heads=4098), "heads"), (dict(dtype=-1), "dtype"),
    (dict(sequences=-1), "sequences"), (dict(sequences=0), "sequence"), (dict(sequences=4), "divide"), (dict(query=None), "query"),
    (dict(value=None), "value"), (dict(log_decay=None), "log_decay"), (dict(scale=math.inf), "scale"), (dict(key_stride=-1), "stride"),
    (dict(key=0x10001), "multiple"), (dict(rows=(1 << 28) - 2, heads=4096, states=4096), "2^31"), (dict(workspace=0x10004), "16 bytes")])
def test_linear_attention_refuses(call, change, text):
    _refused(call, _attention_struct(**change), text)


@pytest.mark.parametrize("call,change,text", [
    ("bagel_linear_attention", dict(out=None), "out"), ("bagel_linear_attention", dict(out_stride=3 * 32 + 15), "overlap"),
    ("bagel_linear_attention", dict(out_head=15), "overlap"), ("bagel_linear_attention", dict(initial=0x20000, final=0x20000), "overlap"),
    ("bagel_linear_attention_grad", dict(d_out=None), "d_out"), ("bagel_linear_attention_grad", dict(d_key_head=31), "overlap"),
    ("bagel_linear_attention_grad", dict(d_final=0x20000, d_initial=0x20010), "overlap"),
    ("bagel_linear_attention_step", dict(), "rows as sequences"), ("bagel_linear_attention_step", dict(sequences=6, state=None), "state"),
    ("bagel_linear_attention_step", dict(sequences=6, out=None), "out"), ("bagel_linear_attention_step", dict(sequences=6, out_stride=0), "overlap"),
    ("bagel_linear_attention_step", dict(sequences=6, value=None), "value"), ("bagel_linear_attention_step", dict(sequences=6, dtype=9), "dtype")])
def test_linear_attention_parts_are_needed(call, change, text):
    _refused(call, _attention_struct(**change), text)


def test_null_arguments_and_sizes_of_work_spaces():
    lib = binding.load()
    for call in ("bagel_layer_norm", "bagel_layer_norm_grad", "bagel_linear_attention", "bagel_linear_attention_grad", "bagel_linear_attention_step"):
        assert getattr(lib, call)(None, None) == binding.EINVAL
    assert lib.bagel_clip_norm(None, 0, None, None) == binding.EINVAL
    assert binding.bagel_layer_norm_workspace(-1, 8) == binding.bagel_layer_norm_workspace(5, 9, 2) == binding.EINVAL
    assert lib.bagel_linear_attention_workspace(None, 0) == lib.bagel_clip_norm_workspace(-1) == binding.EINVAL
    assert binding.bagel_linear_attention_workspace(5, 1, 3, 2, 8, 8) == binding.EINVAL
    assert binding.bagel_linear_attention_workspace(0, 0, 1, 1, 8, 8) >= 0


@pytest.mark.parametrize("change,tensor,text", [
    ({}, dict(dtype=7), "dtype"), (dict(max_norm=-1.0), {}, "max_norm"), (dict(max_norm=NAN), {}, "max_norm"), (dict(eps=0.0), {}, "eps"),
    (dict(norm=None), {}, "norm"), (dict(factor=None), {}, "factor"), (dict(workspace=None), {}, "workspace"), (dict(workspace_bytes=8), {}, "too small"),
    (dict(workspace=0x10004), {}, "16 bytes"), ({}, dict(count=-1), "count"), ({}, dict(grad=None), "null"), ({}, dict(grad=0x10001), "multiple"),
    ({}, dict(out=0x10001), "multiple")])
def test_clip_norm_refuses(change, tensor, text):
    o, t = binding._Clip(), (binding._ClipTensor * 1)()
    o.max_norm, o.eps, o.norm, o.factor, o.workspace, o.workspace_bytes = 1.0, 1e-6, 0x10000, 0x10004, 0x10000, 1 << 20
    t[0].grad, t[0].count, t[0].dtype = 0x10000, 5, 1
    for k, v in change.items():
        setattr(o, k, v)
    for k, v in tensor.items():
        setattr(t[0], k, v)
    lib = binding.load()
    assert lib.bagel_clip_norm(t, 1, C.byref(o), None) == binding.EINVAL
    assert text in lib.bagel_last_error(None).decode()
    assert lib.bagel_clip_norm(None, 1, C.byref(o), None) == lib.bagel_clip_norm(t, -1, C.byref(o), None) == binding.EINVAL


def test_more_structures_are_those_of_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if shutil.which("gcc") is None:
        pytest.skip("gcc not found")
    src = tmp_path / "sizes.c"
    src.write_text("""#include <stdio.h>
#include <stddef.h>
#include "bagel.h"
int main(void) { printf("%zu %zu %zu %zu %zu %zu %zu %zu %zu %d %d\\n", sizeof(bagel_norm), sizeof(bagel_attention), sizeof(bagel_clip_tensor), sizeof(bagel_clip),
offsetof(bagel_norm, workspace), offsetof(bagel_attention, query), offsetof(bagel_attention, state), offsetof(bagel_attention, workspace),
offsetof(bagel_clip, workspace), BAGEL_NORM_MAX_WIDTH, BAGEL_ATTENTION_MAX_WIDTH); return 0; }""")
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", exe, str(src)], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    b = binding
    assert got == [C.sizeof(b._Norm), C.sizeof(b._Attention), C.sizeof(b._ClipTensor), C.sizeof(b._Clip), b._Norm.workspace.offset, b._Attention.query.offset,
                   b._Attention.state.offset, b._Attention.workspace.offset, b._Clip.workspace.offset, b.NORM_MAX_WIDTH, b.ATTENTION_MAX_WIDTH]


def test_binding_refuses_more_before_the_library_is_called():
    x, h = torch.zeros(4, 8), torch.zeros(4, 2, 8)
    ld = torch.zeros(2)
    for call in (lambda: binding.bagel_layer_norm(x, x), lambda: binding.bagel_layer_norm_grad(x, x), lambda: binding.bagel_linear_attention(h, h, h, h, 1, ld),
                 lambda: binding.bagel_linear_attention_grad(h, h, h, h, h, h, h, 1, ld), lambda: binding.bagel_linear_attention_step(h, h, h, h, h, ld)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for bad in (x.double(), None, "text"):
        with pytest.raises(ValueError):
            binding.bagel_layer_norm(bad, x)
    for bad in (None, x, [x.double()], ["text"], 3):
        with pytest.raises(ValueError):
            binding.bagel_clip_norm(bad, 1.0, x, x)
    with pytest.raises(ValueError, match="out"):
        binding.bagel_clip_norm([], 1.0, x, x, out=[x])


@gpu
def test_binding_refuses_more_on_the_gpu():
    x, h, ld = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, 8, device="cuda"), torch.zeros(2, device="cuda")
    for bad in (x[:, :4], x.t().contiguous().t(), x.half(), x.cpu(), x[None], "text"):
        with pytest.raises(ValueError):
            binding.bagel_layer_norm(x, bad)
        with pytest.raises(ValueError):
            binding.bagel_layer_norm_grad(x, bad)
    with pytest.raises(binding.BagelError, match="groups"):
        binding.bagel_layer_norm(x, torch.empty_like(x), groups=3)
    with pytest.raises(ValueError, match="groups"):
        binding.bagel_layer_norm(x, torch.empty_like(x), groups="all")
    with pytest.raises(ValueError, match="weight"):
        binding.bagel_layer_norm(x, torch.empty_like(x), weight=x[0, :4])
    rest = (h, h, h, torch.empty_like(h), 1, ld)
    for place in range(4):
        for bad in (h[:3], h[:, :, :4] if place else h.double(), h.half(), h.cpu(), h[0], "text", h.transpose(1, 2).contiguous().transpose(1, 2)):
            args = list(rest)
            args[place] = bad
            with pytest.raises((ValueError, binding.BagelError)):
                binding.bagel_linear_attention(*args)
    for offsets in (torch.tensor([0, 4], device="cuda"), 2 ** 40, "two", None):
        with pytest.raises(ValueError, match="offsets"):
            binding.bagel_linear_attention(h, h, h, torch.empty_like(h), offsets, ld)
    with pytest.raises(binding.BagelError, match="divide"):
        binding.bagel_linear_attention(h, h, h, torch.empty_like(h), 3, ld)
    with pytest.raises(ValueError, match="log_decay"):
        binding.bagel_linear_attention(h, h, h, torch.empty_like(h), 1, ld[:1])
    with pytest.raises(ValueError, match="scale"):
        binding.bagel_linear_attention(h, h, h, torch.empty_like(h), 1, ld, scale="one")
    with pytest.raises(ValueError, match="initial"):
        binding.bagel_linear_attention(h, h, h, torch.empty_like(h), 1, ld, initial=torch.zeros(1, 2, 8, 7, device="cuda"))
    with pytest.raises(binding.BagelError, match="width"):
        wide = torch.zeros(4, 2, 129, device="cuda")
        binding.bagel_linear_attention(wide, wide, wide, torch.empty_like(wide), 1, ld)
    one = torch.zeros(1, device="cuda")
    with pytest.raises(ValueError, match="tensor 1"):
        binding.bagel_clip_norm([x, x.half()], 1.0, one, torch.zeros_like(one), out=[x, x])
    with pytest.raises(ValueError, match="factor"):
        binding.bagel_clip_norm([x], 1.0, one, ld)
    with pytest.raises(ValueError, match="max_norm"):
        binding.bagel_clip_norm([x], "much", one, torch.zeros_like(one))
