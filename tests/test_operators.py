"""The operators of a policy with memory (block join, gated recurrence, AdamW over many tensors) against plain implementations in
64 bits.

Tolerances.  A result is rounded once to its type: half a unit in the last place of the value, at most 2^-24, 2^-8 or 2^-11 of it (significands of 24, 8 and 11 bits).  Before
that stand sums and products in 32 bits: some forty roundings of 2^-24 on terms no larger than the largest value about, and an
exponential whose argument (up to 10 here) carries a rounding into a relative error of 10 * 2^-24: together below 1e-5 of the largest magnitude.
Where terms cancel it is theirs that counts, and for a sum over rows the sum of theirs."""
import ctypes as C
import math

import pytest
import torch

from paper_2202_13638_amd import binding

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
WORK = 1e-5


def _near(got, want, name, terms=None):
    """`terms`: the sum of the magnitudes that a sum is made of."""
    assert got.shape == want.shape, name
    if want.numel() == 0:
        return
    g, w = got.double().cpu(), want.double().cpu()
    bound = HALF_ULP[got.dtype] * w.abs() * 1.01 + WORK * (w.abs().max() if terms is None else terms.double().cpu())
    if got.dtype == torch.float16:
        bound = bound + 2.0 ** -25                   # its smallest numbers are this far apart, twice
    off = (g - w).abs()
    assert bool((off <= bound).all()), f"{name}: off by {float(off.max()):.3g}, at most {float((off - bound).max()):.3g} too much"


def _normal(shape, seed, dtype=torch.float32, scale=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + mean).to(dtype)


# ------------------------------------------------------------------------------------------------------------- block join
def _act(g, act):
    if act == "none":
        return None, None
    if act == "identity":
        return g, torch.ones_like(g)
    s, r = torch.sigmoid(g), torch.sigmoid(-g)
    return (s, s * r) if act == "logistic" else (g * s, s + g * s * r)


def _ones(t, width):
    return torch.ones(width, dtype=torch.float64) if t is None else t.double()


def _join_ref(branch, resid, gate, act, w, c, u, eps):
    width = (branch if branch is not None else resid).shape[1]
    out = torch.zeros_like(branch.double()) if resid is None else resid.double()
    if branch is not None:
        z = branch.double()
        n = z / torch.sqrt(z.square().mean(1, keepdim=True) + eps) * _ones(w, width)
        a, _ = _act(gate.double() if gate is not None else None, act)
        out = out + _ones(c, width) * (n if a is None else a * n)
    return out, out / torch.sqrt(out.square().mean(1, keepdim=True) + eps) * _ones(u, width)


def _join_inputs(rows, width, dtype, act, seed=0):
    k = 10 * seed
    x = dict(branch=_normal((rows, width), k + 1, dtype, 0.7), resid=_normal((rows, width), k + 2, dtype, 2.0),
             gate=_normal((rows, width), k + 3, dtype, 1.5) if act != "none" else None,
             post_weight=_normal((width,), k + 4, scale=0.2, mean=1.0), scale=_normal((width,), k + 5, scale=0.2, mean=0.3),
             pre_weight=_normal((width,), k + 6, scale=0.2, mean=1.0))
    return x


def _cuda(d):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


JOIN_SIZES = [(1, 1), (3, 2), (2, 63), (5, 64), (4, 65), (7, 255), (9, 256), (3, 777), (33, 1000), (2, 1024), (2, 1026), (5, 2048), (3, 2056),
              (2, 4096), (3, 5001), (2, 8192), (2, 16384), (1, 16383)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", JOIN_SIZES)
def test_join_and_its_gradient(rows, width, dtype):
    t = TYPES[dtype]
    act = ["silu", "logistic", "identity", "none"][(rows + width) % 4]
    x = _join_inputs(rows, width, t, act)
    g = _cuda(x)
    out, normed = (torch.full((rows, width), float("nan"), dtype=t, device="cuda") for _ in range(2))
    rest = dict(act=act, eps=1e-5, **{k: g[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
    binding.bagel_block_join(g["branch"], g["resid"], out, normed, **rest)
    want = _join_ref(x["branch"], x["resid"], x["gate"], act, x["post_weight"], x["scale"], x["pre_weight"], 1e-5)
    _near(out, want[0], "out")
    _near(normed, want[1], "normed")
    d_out, d_normed = _normal((rows, width), 7, t), _normal((rows, width), 8, t)
    _join_grad_case(x, g, out, d_out, d_normed, act, 1e-5)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(70001, 40), (17, 100), (15, 8), (16, 9), (33, 121), (2, 4), (20003, 64)])
def test_join_of_short_rows(rows, width, dtype):
    """Rows that take a part of a wave, and more of them than there are places."""
    test_join_and_its_gradient(rows, width, dtype)


def _join_grad_ref(x, out, d_out, d_normed, act, eps):
    """Gradients, and the sums of magnitudes of those of the vectors, from the formulas in 64 bits at the stored `out`."""
    width = out.shape[1]
    w, c, u = (_ones(x[k], width) for k in ("post_weight", "scale", "pre_weight"))
    o = out.double().cpu()
    dy = torch.zeros_like(o) if d_normed is None else d_normed.double()

    def norm_grad(d, z):
        r = torch.sqrt(z.square().mean(1, keepdim=True) + eps)
        return (d - z / r * (d * z / r).mean(1, keepdim=True)) / r, z / r

    d, n_out = norm_grad(dy * u, o)
    dx = d if d_out is None else d + d_out.double()
    r = {"d_resid": dx, "d_pre_weight": (dy * n_out).sum(0)}
    # what dx is the sum of: its parts may cancel (of a row of one entry they do)
    parts = (0 if d_out is None else d_out.double().abs()) + d.abs() + 2 * (dy * u / torch.sqrt(o.square().mean(1, keepdim=True) + eps)).abs()
    terms = {"d_pre_weight": (dy * n_out).abs().sum(0), "d_resid": parts.max()}
    if x["branch"] is not None:
        a, da = _act(x["gate"].double() if x["gate"] is not None else None, act)
        a = torch.ones_like(o) if a is None else a
        r["d_branch"], n = norm_grad(dx * c * w * a, x["branch"].double())
        if act != "none":
            r["d_gate"] = dx * c * w * n * da
        r["d_post_weight"], r["d_scale"] = (dx * c * a * n).sum(0), (dx * w * a * n).sum(0)
        terms["d_post_weight"], terms["d_scale"] = (parts * c * a * n).abs().sum(0), (parts * w * a * n).abs().sum(0)
        rz = 1 / torch.sqrt(x["branch"].double().square().mean(1, keepdim=True) + eps)
        terms["d_branch"] = 2 * (parts * c * w * a * rz).abs().max()
        if act != "none":
            terms["d_gate"] = (parts * c * w * n * da).abs().max()
    return r, terms


def _join_grad_case(x, g, out, d_out, d_normed, act, eps, **layout):
    want, terms = _join_grad_ref(x, out, d_out, d_normed, act, eps)
    got = {k: torch.full(v.shape, float("nan"), dtype=out.dtype if v.dim() == 2 else torch.float32, device="cuda") for k, v in want.items()}
    binding.bagel_block_join_grad(g["branch"], out, None if d_out is None else d_out.cuda(), None if d_normed is None else d_normed.cuda(),
                                  act=act, eps=eps, **{k: g[k] for k in ("gate", "post_weight", "scale", "pre_weight")}, **got)
    for k, v in want.items():
        extra = terms.get(k)
        _near(got[k], v, k, terms=None if extra is None else extra + 1e-30)
    return got


@gpu
@pytest.mark.parametrize("act", ["none", "identity", "logistic", "silu"])
@pytest.mark.parametrize("left_out", ["nothing", "vectors", "branch", "resid", "out", "normed", "d_out", "d_normed"])
def test_join_with_parts_left_out(act, left_out):
    rows, width, t = 6, 72, torch.float32
    x = _join_inputs(rows, width, t, act)
    if left_out == "vectors":
        x["post_weight"] = x["scale"] = x["pre_weight"] = None
    elif left_out == "branch":
        x["branch"] = x["gate"] = None
        act = "none"
    elif left_out == "resid":
        x["resid"] = None
    g = _cuda(x)
    out, normed = torch.zeros(rows, width, device="cuda"), torch.zeros(rows, width, device="cuda")
    rest = dict(act=act, **{k: g[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
    binding.bagel_block_join(g["branch"], g["resid"], None if left_out == "out" else out, None if left_out == "normed" else normed, **rest)
    want = _join_ref(x["branch"], x["resid"], x["gate"], act, x["post_weight"], x["scale"], x["pre_weight"], 1e-6)
    if left_out != "out":
        _near(out, want[0], "out")
    if left_out != "normed":
        _near(normed, want[1], "normed")
    d_out = None if left_out == "d_out" else _normal((rows, width), 7)
    d_normed = None if left_out == "d_normed" else _normal((rows, width), 8)
    _join_grad_case(x, g, want[0].float().cuda(), d_out, d_normed, act, 1e-6)


@gpu
def test_join_of_zero_rows_of_zeros_and_of_extreme_gates():
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    d = torch.full((64,), 5.0, device="cuda")
    binding.bagel_block_join(e, e.clone(), e.clone(), e.clone())
    binding.bagel_block_join_grad(e, e.clone(), e.clone(), e.clone(), d_post_weight=d, post_weight=w)
    assert not d.any()                                              # a sum over nothing
    z = torch.zeros(3, 64, device="cuda")
    out, normed = torch.full_like(z, 7), torch.full_like(z, 7)
    binding.bagel_block_join(z, z, out, normed)
    assert not out.any() and not normed.any()
    grads = [torch.full_like(z, 7) for _ in range(2)]
    binding.bagel_block_join_grad(z, z, z + 1, z + 1, d_branch=grads[0], d_resid=grads[1])
    assert all(torch.isfinite(v).all() for v in grads)
    gate = torch.tensor([-1e4, 1e4, -200.0, 200.0, -88.0, 88.0, 0.0, 1.0], device="cuda").repeat(8)[None]
    for act in ("logistic", "silu"):
        x = dict(branch=torch.ones(1, 64), gate=gate.cpu(), resid=torch.zeros(1, 64), post_weight=None, scale=None, pre_weight=None)
        g = _cuda(x)
        out = torch.empty(1, 64, device="cuda")
        binding.bagel_block_join(g["branch"], g["resid"], out, gate=g["gate"], act=act)
        want = _join_ref(x["branch"], x["resid"], x["gate"], act, None, None, None, 1e-6)[0]
        _near(out, want, act)
        _join_grad_case(x, g, out, _normal((1, 64), 3), _normal((1, 64), 4), act, 1e-6)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,stride,width", [(0, 640, 512), (8, 1040, 512), (1, 515, 512), (3, 131, 64), (0, 200, 77), (4, 260, 256), (2, 2050, 2048)])
def test_join_of_strided_rows(start, stride, width, dtype):
    t, rows, act = TYPES[dtype], 5, "silu"
    x = _join_inputs(rows, width, t, act)

    def strided(v, i):                                              # a window into a larger buffer, another one for each
        buffer = torch.full((rows * (stride + 16 * i) + start + width,), float("nan"), dtype=t, device="cuda")
        view = buffer[start:].as_strided((rows, width), (stride + 16 * i, 1), start)
        if v is not None:
            view.copy_(v)
        return view, buffer

    g = {k: (strided(v, i)[0] if v.dim() == 2 else v.cuda()) for i, (k, v) in enumerate(x.items())}
    (out, whole), (normed, _) = strided(None, 1), strided(None, 2)
    rest = dict(act=act, **{k: g[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
    binding.bagel_block_join(g["branch"], g["resid"], out, normed, **rest)
    same = {k: v.contiguous() if v.dim() == 2 else v for k, v in g.items()}
    want = _join_ref(x["branch"], x["resid"], x["gate"], act, x["post_weight"], x["scale"], x["pre_weight"], 1e-6)
    _near(out, want[0], "out")
    _near(normed, want[1], "normed")
    assert int(torch.isfinite(whole).sum()) == rows * width         # nothing was written beside the rows
    d_out, d_normed = strided(_normal((rows, width), 7, t), 0)[0], strided(_normal((rows, width), 8, t), 3)[0]
    got = {k: strided(None, i)[0] for i, k in enumerate(("d_branch", "d_gate", "d_resid"))}
    vec = {k: torch.empty(width, device="cuda") for k in ("d_post_weight", "d_scale", "d_pre_weight")}
    binding.bagel_block_join_grad(g["branch"], out, d_out, d_normed, **rest, **got, **vec)
    expect, terms = _join_grad_ref(x, out.contiguous(), d_out.cpu(), d_normed.cpu(), act, 1e-6)
    for k, v in {**got, **vec}.items():
        _near(v, expect[k], k, terms=terms.get(k))
    del same


@gpu
def test_join_in_place_and_repeated():
    rows, width, act = 700, 520, "silu"
    x = _cuda(_join_inputs(rows, width, torch.bfloat16, act))
    rest = dict(act=act, **{k: x[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
    out, place = torch.empty_like(x["resid"]), x["resid"].clone()
    binding.bagel_block_join(x["branch"], x["resid"], out, **rest)
    binding.bagel_block_join(x["branch"], place, place, **rest)
    assert torch.equal(out, place)
    d_out, d_normed = (_normal((rows, width), i, torch.bfloat16).cuda() for i in (7, 8))
    runs = []
    for k in range(3):
        d = d_out.clone()
        vec = {n: torch.empty(width, device="cuda") for n in ("d_post_weight", "d_scale", "d_pre_weight")}
        d_resid = d if k == 2 else torch.empty_like(d)
        binding.bagel_block_join_grad(x["branch"], out, d, d_normed, **rest, d_resid=d_resid, **vec)
        runs.append([d_resid, *vec.values()])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


@gpu
def test_join_rows_beyond_32_bits():
    """Rows that begin past 2^31 and 2^32 entries into their buffer."""
    width, stride, rows = 256, 1 << 28, 20
    x = _join_inputs(rows, width, torch.bfloat16, "none")
    big = torch.empty(stride * (rows - 1) + width, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((rows, width), (stride, 1))
    view.copy_(x["resid"])
    g = _cuda(x)
    binding.bagel_block_join(g["branch"], view, view, scale=g["scale"])
    _near(view.contiguous(), _join_ref(x["branch"], x["resid"], None, "none", None, x["scale"], None, 1e-6)[0], "out")


@gpu
def test_a_nan_stays_in_its_row():
    x = _cuda(_join_inputs(9, 320, torch.bfloat16, "silu"))
    rest = dict(act="silu", **{k: x[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
    a, b = torch.empty_like(x["resid"]), torch.empty_like(x["resid"])
    binding.bagel_block_join(x["branch"], x["resid"], None, a, **rest)
    x["branch"][4, 7] = float("nan")
    binding.bagel_block_join(x["branch"], x["resid"], None, b, **rest)
    others = [i for i in range(9) if i != 4]
    assert torch.equal(a[others], b[others]) and torch.isnan(b[4]).all()


# ------------------------------------------------------------------------------------------------------ gated recurrence
def _recurrence_ref(value, forget, at, bias, initial, d_hidden, d_final):
    """Step by step in 64 bits; rows behind the last sequence are zero."""
    x, f = value.double(), forget.double() + (0 if bias is None else bias.double())
    q, a = torch.sigmoid(-f), torch.sigmoid(f)
    n, width = len(at) - 1, x.shape[1]
    h0 = torch.zeros(n, width, dtype=torch.float64) if initial is None else initial.double()
    dl = torch.zeros(n, width, dtype=torch.float64) if d_final is None else d_final.double()
    h, dx, df = (torch.zeros_like(x) for _ in range(3))
    final, d0 = h0.clone(), dl.clone()
    for i in range(n):
        if at[i] == at[i + 1]:
            continue
        state, before = h0[i], {}
        for t in range(at[i], at[i + 1]):
            before[t] = state
            state = state * a[t] + q[t] * x[t]
            h[t] = state
        final[i], c = state, dl[i]
        for t in range(at[i + 1] - 1, at[i] - 1, -1):
            g = d_hidden[t].double() + c
            dx[t], df[t], c = q[t] * g, (before[t] - x[t]) * q[t] * a[t] * g, a[t] * g
        d0[i] = c
    return dict(hidden=h, final=final, d_value=dx, d_forget=df, d_initial=d0, d_bias=df.sum(0)), df.abs().sum(0)


def _run_recurrence(value, forget, at, bias, initial, d_hidden, d_final, want=(), offsets=None):
    rows, width = value.shape
    n = len(at) - 1
    offsets = torch.tensor(at, dtype=torch.int32).cuda() if offsets is None else offsets
    nan = float("nan")
    like = lambda: torch.full((rows, width), nan, dtype=value.dtype, device="cuda")  # noqa: E731
    r = dict(hidden=like(), final=torch.full((n, width), nan, device="cuda"), d_value=like(), d_forget=like(),
             d_initial=torch.full((n, width), nan, device="cuda"), d_bias=torch.full((width,), nan, device="cuda"))
    carry = torch.full((binding.bagel_recurrence_carry_rows(rows), width), nan, device="cuda")
    binding.bagel_recurrence(value, forget, r["hidden"], offsets, bias=bias, initial=initial, final=r["final"], carry=carry)
    binding.bagel_recurrence_grad(value, forget, d_hidden, r["d_value"], r["d_forget"], offsets, carry, bias=bias, initial=initial,
                                  d_final=d_final, d_initial=r["d_initial"], d_bias=r["d_bias"])
    return r


LENGTHS = {
    "one": [1], "two": [2], "span": [128], "span+1": [129], "ones": [1] * 70, "empty between": [0, 5, 0, 0, 130, 0, 1, 0],
    "all empty": [0, 0, 0], "spans": [127, 128, 129, 1, 256, 255], "long": [1500], "longer": [3000, 2, 700], "short": [3, 7, 16, 31, 33, 64, 15, 17] * 6,
}


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 2, 64, 77, 130, 260])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_recurrence_and_its_gradient(lengths, width, dtype):
    t, at = TYPES[dtype], [0]
    for n in LENGTHS[lengths]:
        at.append(at[-1] + n)
    rows, n, bare = at[-1], len(at) - 1, width == 130               # one width without what may be left out
    x, f, dh = (_normal((rows, width), i, t) for i in (1, 2, 3))
    bias, h0, dl = (_normal((width,), 4, mean=2.0), _normal((n, width), 5), _normal((n, width), 6)) if not bare else (None, None, None)
    want, terms = _recurrence_ref(x, f, at, bias, h0, dh, dl)
    got = _run_recurrence(x.cuda(), f.cuda(), at, *(None if v is None else v.cuda() for v in (bias, h0)), dh.cuda(), None if dl is None else dl.cuda())
    for k, v in want.items():
        _near(got[k], v, k, terms=terms + 1e-30 if k == "d_bias" else None)


@gpu
@pytest.mark.parametrize("width", [70, 131])
def test_recurrence_over_many_spans_gives_the_same_bits_every_time(width):
    """Sequences over several blocks of 32 spans, where a span's state comes from others that run beside it."""
    at = [0, 9000, 9001, 14100]
    x, f, dh = (_normal((at[-1], width), i, torch.bfloat16).cuda() for i in (1, 2, 3))
    bias, h0, dl = _normal((width,), 4, mean=3.0).cuda(), _normal((3, width), 5).cuda(), _normal((3, width), 6).cuda()
    runs = [_run_recurrence(x, f, at, bias, h0, dh, dl) for _ in range(4)]
    for other in runs[1:]:
        for k, v in runs[0].items():
            assert torch.equal(v, other[k]), k
    want, terms = _recurrence_ref(*(t.cpu() for t in (x, f)), at, *(t.cpu() for t in (bias, h0, dh, dl)))
    for k, v in want.items():
        _near(runs[0][k], v, k, terms=terms if k == "d_bias" else None)


@gpu
@pytest.mark.parametrize("rows, width, dtype", [(14100, 600, "bf16"), (14100, 300, "f32"), (70000, 33, "bf16"), (70000, 3, "f32"), (4096, 70, "f16"), (4097, 70, "f16")])
def test_recurrence_over_blocks_of_spans(rows, width, dtype):
    """Few channels and many, over more than two of the largest blocks of spans, and at the rows from which blocks of blocks are used."""
    at = [0, 2000, 2000, rows - 7, rows]
    x, f, dh = (_normal((rows, width), i, TYPES[dtype]).cuda() for i in (1, 2, 3))
    bias, h0, dl = _normal((width,), 4, mean=5.0).cuda(), _normal((4, width), 5).cuda(), _normal((4, width), 6).cuda()
    got, again = (_run_recurrence(x, f, at, bias, h0, dh, dl) for _ in range(2))
    want, terms = _recurrence_ref(*(t.cpu() for t in (x, f)), at, *(t.cpu() for t in (bias, h0, dh, dl)))
    for k, v in want.items():
        assert torch.equal(got[k], again[k]), k
        _near(got[k], v, k, terms=terms if k == "d_bias" else None)


@gpu
@pytest.mark.parametrize("count", [62, 63, 64, 65, 700, 5000])
def test_recurrence_of_many_short_sequences(count):
    """Numbers of sequences at which the search for a row's sequence takes one look, two and three; a third of them are empty."""
    g = torch.Generator().manual_seed(count)
    n = torch.randint(0, 9, (count,), generator=g) * (torch.rand(count, generator=g) > 0.33)
    at = [0] + torch.cumsum(n, 0).tolist()
    width = 10
    x, f, dh = (_normal((at[-1], width), i).cuda() for i in (1, 2, 3))
    bias, h0, dl = _normal((width,), 4).cuda(), _normal((count, width), 5).cuda(), _normal((count, width), 6).cuda()
    got = _run_recurrence(x, f, at, bias, h0, dh, dl)
    want, terms = _recurrence_ref(*(t.cpu() for t in (x, f)), at, *(t.cpu() for t in (bias, h0, dh, dl)))
    for k, v in want.items():
        _near(got[k], v, k, terms=terms if k == "d_bias" else None)


@gpu
def test_recurrence_of_every_kind_of_nan():
    """What is published of a span is told from nothing by a bit pattern: no NaN of the inputs may look like it."""
    rows, width = 5000, 64
    x, f, dh = (_normal((rows, width), i).cuda() for i in (1, 2, 3))
    for k, bits in enumerate((-1, 0x7FFFFFFF, 0x7FC00000, -4194304, 0x7F800001)):
        nan = torch.tensor([bits], dtype=torch.int32, device="cuda").view(torch.float32)
        for t in (x, f, dh):
            t[100 + 300 * k, k] = nan[0]
    r = _run_recurrence(x, f, [0, rows], None, None, dh, None)
    assert torch.isnan(r["hidden"][-1, :5]).all() and torch.isfinite(r["hidden"][:, 5:]).all()
    assert torch.isfinite(r["d_value"][:, 5:]).all() and torch.isnan(r["d_initial"][0, :5]).all()


@gpu
def test_recurrence_rows_beyond_32_bits():
    rows, width, stride = 600, 6, 1 << 23
    big = torch.empty(stride * (rows - 1) + 6 * width, dtype=torch.bfloat16, device="cuda")
    v = [big.as_strided((rows, width), (stride, 1), i * width) for i in range(6)]
    x, f, dh = (_normal((rows, width), i, torch.bfloat16) for i in (1, 2, 3))
    for to, src in zip(v, (x, f, dh)):
        to.copy_(src)
    carry = torch.empty(binding.bagel_recurrence_carry_rows(rows), width, device="cuda")
    binding.bagel_recurrence(v[0], v[1], v[3], 1, carry=carry)
    binding.bagel_recurrence_grad(v[0], v[1], v[2], v[4], v[5], 1, carry)
    want, _ = _recurrence_ref(x, f, [0, rows], None, None, dh, None)
    for t, k in zip(v[3:], ("hidden", "d_value", "d_forget")):
        _near(t.contiguous(), want[k], k)


@gpu
def test_recurrence_equal_lengths_without_offsets():
    rows, n, width = 7 * 93, 7, 66
    x, f, dh = (_normal((rows, width), i).cuda() for i in (1, 2, 3))
    h0, dl = _normal((n, width), 5).cuda(), _normal((n, width), 6).cuda()
    at = [93 * i for i in range(n + 1)]
    a, b = _run_recurrence(x, f, at, None, h0, dh, dl), _run_recurrence(x, f, at, None, h0, dh, dl, offsets=n)
    assert all(torch.equal(a[k], b[k]) for k in a)


@gpu
@pytest.mark.parametrize("tail", [1, 64, 129, 300])
def test_rows_behind_the_last_sequence_are_not_used(tail):
    at, width = [0, 200, 200, 331], 70
    rows = at[-1] + tail
    x, f, dh = (_normal((rows, width), i, torch.bfloat16) for i in (1, 2, 3))
    for v in (x, f, dh):
        v[at[-1]:] = float("nan")
    bias, h0, dl = _normal((width,), 4), _normal((3, width), 5), _normal((3, width), 6)
    want, terms = _recurrence_ref(x[:at[-1]], f[:at[-1]], at, bias, h0, dh[:at[-1]], dl)
    got = _run_recurrence(x.cuda(), f.cuda(), at, bias.cuda(), h0.cuda(), dh.cuda(), dl.cuda())
    for k in ("hidden", "d_value", "d_forget"):
        assert not got[k][at[-1]:].any()                            # neither a number nor NaN
        got[k] = got[k][:at[-1]]
    for k, v in want.items():
        _near(got[k], v, k, terms=terms if k == "d_bias" else None)


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_sequence(bad):
    at, width = [0, 300, 710, 711, 900], 96
    x, f, dh = (_normal((at[-1], width), i).cuda() for i in (1, 2, 3))
    h0, dl = _normal((4, width), 5).cuda(), _normal((4, width), 6).cuda()
    a = _run_recurrence(x, f, at, None, h0, dh, dl)
    x[500, 3], dh[600, 5], f[350, 9] = bad, bad, float("nan")
    b = _run_recurrence(x, f, at, None, h0, dh, dl)
    rows = torch.tensor([i for i in range(at[-1]) if not 300 <= i < 710], device="cuda")
    for k in ("hidden", "d_value", "d_forget"):
        assert torch.equal(a[k][rows], b[k][rows]), k
    for k in ("final", "d_initial"):
        assert torch.equal(a[k][[0, 2, 3]], b[k][[0, 2, 3]]), k
    assert not torch.isfinite(b["hidden"][709, 3]) and torch.isnan(b["hidden"][709, 9])


@gpu
def test_recurrence_of_closed_and_open_gates():
    """A forget gate of +infinity keeps the state to the last bit, one of -infinity takes the value (to a rounding of their difference)."""
    rows, width = 700, 64
    x = _normal((rows, width), 1).cuda()
    h0, keep = _normal((1, width), 2).cuda(), torch.full((rows, width), float("inf"), device="cuda")
    for f, want in ((keep, h0.expand(rows, width)), (-keep, x), (keep.clamp(max=1e4), h0.expand(rows, width)), (-keep.clamp(max=1e4), x)):
        r = _run_recurrence(x, f, [0, rows], None, h0, torch.ones_like(x), None)
        if f[0, 0] > 0:
            assert torch.equal(r["hidden"], want) and torch.equal(r["final"], want[-1:])
        _near(r["hidden"], want.cpu(), "hidden")
        _near(r["final"], want[-1:].cpu(), "final")
        assert all(torch.isfinite(r[k]).all() for k in ("d_value", "d_forget", "d_initial", "d_bias"))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,stride,width", [(0, 256, 128), (1, 301, 128), (2, 258, 130), (0, 100, 33), (8, 1024, 512)])
def test_recurrence_of_strided_rows(start, stride, width, dtype):
    t, at = TYPES[dtype], [0, 140, 143, 400]
    rows = at[-1]
    x, f, dh = (_normal((rows, width), i, t).cuda() for i in (1, 2, 3))
    h0, bias = _normal((3, width), 5).cuda(), _normal((width,), 4).cuda()
    want, _ = _recurrence_ref(x.cpu(), f.cpu(), at, bias.cpu(), h0.cpu(), dh.cpu(), None)
    buffers = [torch.full((rows * stride + start + width,), float("nan"), dtype=t, device="cuda") for _ in range(6)]
    v = [b.as_strided((rows, width), (stride, 1), start) for b in buffers]
    for to, src in zip(v, (x, f, dh)):
        to.copy_(src)
    offsets = torch.tensor(at, dtype=torch.int32).cuda()
    carry = torch.empty(binding.bagel_recurrence_carry_rows(rows), width, device="cuda")
    binding.bagel_recurrence(v[0], v[1], v[3], offsets, bias=bias, initial=h0, carry=carry)
    binding.bagel_recurrence_grad(v[0], v[1], v[2], v[4], v[5], offsets, carry, bias=bias, initial=h0)
    for b, got, k in zip(buffers[3:], v[3:], ("hidden", "d_value", "d_forget")):
        _near(got, want[k], k)
        assert int(torch.isfinite(b).sum()) == rows * width


@gpu
def test_recurrence_step_is_the_sequence_one_row_at_a_time():
    n, steps, width = 5, 40, 129
    x, f = _normal((n, steps, width), 1, torch.bfloat16).cuda(), _normal((n, steps, width), 2, torch.bfloat16).cuda()
    bias, h0 = _normal((width,), 3).cuda(), _normal((n, width), 4).cuda()
    hidden = torch.empty(n * steps, width, dtype=torch.bfloat16, device="cuda")
    final, state = torch.empty_like(h0), h0.clone()
    binding.bagel_recurrence(x.view(-1, width), f.view(-1, width), hidden, n, bias=bias, initial=h0, final=final)
    for t in range(steps):
        y = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
        binding.bagel_recurrence_step(x[:, t], f[:, t], state, y if t % 2 else None, bias=bias)
        if t % 2:
            _near(y, _step_want(x, f, bias, h0, t), f"step {t}")
    want = _step_want(x, f, bias, h0, steps - 1)
    _near(state, want, "state")
    _near(final, want, "final")


def _step_want(x, f, bias, h0, t):
    h = h0.double()
    for i in range(t + 1):
        q = torch.sigmoid(-(f[:, i].double() + bias.double()))
        h = h + q * (x[:, i].double() - h)
    return h.cpu()


@gpu
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 64), (3, 1000), (300, 37), (70, 512), (0, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence_step(rows, width, dtype):
    t = TYPES[dtype]
    x, f, state = _normal((rows, width), 1, t), _normal((rows, width), 2, t), _normal((rows, width), 3)
    bias = _normal((width,), 4)
    want = _step_want(x[:, None], f[:, None], bias, state, 0)
    s, y = state.cuda(), torch.empty(rows, width, dtype=t, device="cuda")
    binding.bagel_recurrence_step(x.cuda(), f.cuda(), s, y, bias=bias.cuda())
    _near(s, want, "state")
    _near(y, want, "hidden")


@gpu
def test_gradients_against_differences():
    """L = <weights, outputs> of the kernels themselves, differentiated along random directions.  Inputs move by 1e-2 of a
    normal direction: third derivatives leave 1e-4 of the slope, rounding (2^-24 on sums of some thousand terms) less."""
    def slope(f, at, way, h=1e-2):
        up, down = ([p + s * h * d for p, d in zip(at, way)] for s in (1, -1))
        return (f(*up) - f(*down)) / (2 * h)

    at, width = [0, 140, 141, 400], 48
    args = [_normal((400, width), 1).cuda(), _normal((400, width), 2).cuda(), _normal((width,), 3).cuda(), _normal((3, width), 4).cuda()]
    way = [_normal(p.shape, 10 + i).cuda() for i, p in enumerate(args)]
    dh, dl = _normal((400, width), 20).cuda(), _normal((3, width), 21).cuda()

    def loss(x, f, b, h0):
        r = _run_recurrence(x, f, at, b, h0, dh, dl)
        return float((r["hidden"].double() * dh).sum() + (r["final"].double() * dl).sum())

    r = _run_recurrence(args[0], args[1], at, args[2], args[3], dh, dl)
    for i, k in enumerate(("d_value", "d_forget", "d_bias", "d_initial")):
        only = [w if j == i else torch.zeros_like(w) for j, w in enumerate(way)]
        want = slope(loss, args, only)
        got = float((r[k].double() * way[i]).sum())
        size = float((r[k].double().norm() * way[i].double().norm()))
        assert abs(got - want) <= 1e-3 * size, (k, got, want)

    rows, width = 12, 320
    names = ("branch", "resid", "gate", "post_weight", "scale", "pre_weight")
    x = _cuda(_join_inputs(rows, width, torch.float32, "silu"))
    way = {k: _normal(x[k].shape, 30 + i).cuda() for i, k in enumerate(names)}
    d_out, d_normed = _normal((rows, width), 40).cuda(), _normal((rows, width), 41).cuda()

    def join(y):
        out, normed = torch.empty_like(d_out), torch.empty_like(d_out)
        binding.bagel_block_join(y["branch"], y["resid"], out, normed, act="silu", **{k: y[k] for k in names[2:]})
        return out, normed

    out, _ = join(x)
    r = {"d_" + k: torch.empty_like(x[k]) for k in names}
    binding.bagel_block_join_grad(x["branch"], out, d_out, d_normed, act="silu", **{k: x[k] for k in names[2:]}, **r)
    for k in names:
        def loss(v):
            o, y = join({**x, k: v})
            return float((o.double() * d_out).sum() + (y.double() * d_normed).sum())
        want, got = slope(loss, [x[k]], [way[k]]), float((r["d_" + k].double() * way[k]).sum())
        assert abs(got - want) <= 1e-3 * float(r["d_" + k].double().norm() * way[k].double().norm()), (k, got, want)


# ------------------------------------------------------------------------------------------------------------------ AdamW
SHAPES = [(1,), (2,), (255,), (256,), (257,), (33, 77), (1024,), (0,), (3, 5, 7), (4096,), (5001,)]


def _adamw_ref(p, g, m, v, step, lr, b1, b2, eps, wd):
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = p - lr * wd * p - lr * (m / (1 - b1 ** step)) / (torch.sqrt(v / (1 - b2 ** step)) + eps)
    return p, m, v


@gpu
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("copy", [None, "f32", "bf16", "f16"])
@pytest.mark.parametrize("step", [1, 7, 100000])
def test_adamw(step, copy, grad):
    p = [_normal(s, i) for i, s in enumerate(SHAPES)]
    g = [_normal(s, 20 + i, TYPES[grad], 0.01) for i, s in enumerate(SHAPES)]
    m, v = [_normal(s, 40 + i, scale=1e-3) for i, s in enumerate(SHAPES)], [_normal(s, 60 + i, scale=1e-2).square() for i, s in enumerate(SHAPES)]
    decay = [0.1 if len(s) > 1 else 0.0 for s in SHAPES]
    scale = torch.tensor([0.25])
    c = None if copy is None else [torch.empty(s, dtype=TYPES[copy], device="cuda") for s in SHAPES]
    d = [[t.cuda() for t in x] for x in (p, g, m, v)]
    binding.bagel_adamw_step(*d, step, copy=c, lr=1e-2, beta1=0.8, beta2=0.99, eps=1e-6, weight_decay=decay, grad_scale=scale.cuda())
    for i in range(len(SHAPES)):
        want = _adamw_ref(p[i].double(), g[i].double() * 0.25, m[i].double(), v[i].double(), step, 1e-2, 0.8, 0.99, 1e-6, decay[i])
        for k, name in enumerate(("p", "m", "v")):
            _near(d[(0, 2, 3)[k]][i], want[k], f"{name} of {SHAPES[i]}")
        if c is not None:
            assert torch.equal(c[i], d[0][i].to(TYPES[copy]))


@gpu
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_adamw_at_odd_starts(shift):
    """Tensors at any multiple of their type; what stands beside them stays."""
    n = 3001

    def at(t, dtype=None):
        b = torch.full((n + 64,), 3.0, device="cuda").to(t.dtype)
        b[shift:shift + n] = t.cuda()
        return b, b[shift:shift + n]

    for bits in (32, 8):
        p, g = _normal((n,), 1), _normal((n,), 2, torch.bfloat16)
        if bits == 32:
            m, v, extra = _normal((n,), 3), _normal((n,), 4).square(), {}
        else:
            m, v = _normal((n,), 3, scale=100).clamp(-448, 448).to(torch.float8_e4m3fn), _normal((n,), 4, scale=50).abs().to(torch.float8_e4m3fn)
            s = torch.full((12,), 1e-3)
            extra = lambda: dict(m_scale=[s.cuda()], v_scale=[s.cuda()])  # noqa: E731
        plain = [t.cuda() for t in (p, g, m, v)]
        odd = [at(t) for t in (p, g, m, v)]
        one, two = ({}, {}) if bits == 32 else (extra(), extra())
        binding.bagel_adamw_step(*[[t] for t in plain], 5, **one)
        binding.bagel_adamw_step(*[[t[1]] for t in odd], 5, **two)
        for a, (whole, b) in zip(plain, odd):
            assert torch.equal(a.view(torch.uint8), b.contiguous().view(torch.uint8))
            beside = torch.cat([whole[:shift], whole[shift + n:]]).float()
            assert bool((beside == 3.0).all())
        if bits == 8:
            assert torch.equal(one["m_scale"][0], two["m_scale"][0]) and torch.equal(one["v_scale"][0], two["v_scale"][0])


@gpu
def test_adamw_of_many_tensors_is_each_on_its_own():
    shapes = [(1 + 37 * i % 1000,) for i in range(150)]
    p, g = [_normal(s, i).cuda() for i, s in enumerate(shapes)], [_normal(s, 200 + i).cuda() for i, s in enumerate(shapes)]
    m, v = [torch.zeros(s, device="cuda") for s in shapes], [torch.zeros(s, device="cuda") for s in shapes]
    one = [[t.clone() for t in x] for x in (p, m, v)]
    binding.bagel_adamw_step(p, g, m, v, 1)
    for i in range(len(shapes)):
        binding.bagel_adamw_step([one[0][i]], [g[i]], [one[1][i]], [one[2][i]], 1)
    assert all(torch.equal(a, b) for x, y in zip((p, m, v), one) for a, b in zip(x, y))


def _values(codes, scale):
    n = codes.numel()
    return (codes.reshape(-1).double().cpu() * scale.double().cpu().repeat_interleave(256)[:n])


@gpu
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_adamw_in_8_bits(shape, grad):
    """Codes lie on either side of the value they stand for: within a code's distance, an eighth of its power of two or, for the
    smallest, 2^-9 of the scale."""
    n = math.prod(shape)
    blocks = -(-n // 256)
    p, g = _normal(shape, 1), _normal(shape, 2, TYPES[grad], 0.1)
    m = _normal(shape, 3, scale=100).clamp(-448, 448).to(torch.float8_e4m3fn)
    r = _normal(shape, 4, scale=100).abs().clamp(2, 448).to(torch.float8_e4m3fn)
    sm, sv = _normal((blocks,), 5).abs() * 1e-3 + 1e-4, _normal((blocks,), 6).abs() * 1e-3 + 1e-4
    d = [t.cuda() for t in (p, g, m, r)]
    dm, dv = sm.cuda(), sv.cuda()
    binding.bagel_adamw_step(*[[t] for t in d], 50, m_scale=[dm], v_scale=[dv], lr=1e-2, weight_decay=0.0)
    want = _adamw_ref(p.double().reshape(-1), g.double().reshape(-1), _values(m, sm), _values(r, sv) ** 2, 50, 1e-2, 0.9, 0.999, 1e-8, 0.0)
    _near(d[0].reshape(-1), want[0], "p")
    for codes, scale, x in ((d[2], dm, want[1]), (d[3], dv, want[2].sqrt())):
        if n == 0:
            continue
        each = torch.arange(n) // 256
        top = torch.zeros(blocks, dtype=torch.float64).scatter_reduce(0, each, x.abs(), "amax")
        _near(scale, top / 448, "scale")
        at = (top / 448)[each]
        step = torch.where(x.abs() / at < 2 ** -6, 2.0 ** -9, 2.0 ** (torch.floor(torch.log2((x.abs() / at).clamp(min=2 ** -6))) - 3)) * at
        off = (_values(codes, scale) - x).abs()
        assert bool((off <= step * (1 + 1e-4)).all()), float((off / step).max())
        assert bool(((codes.float().cpu().reshape(-1) != 0) | (x == 0) | (codes is d[2])).all())     # no root becomes zero
        assert bool((codes.float().abs().max() == 448.0))


@gpu
def test_adamw_in_8_bits_keeps_means():
    """Rounding by chance: over places that hold the same value, and over updates, the mean of the codes is the value.  With n = 2^16 places
    the mean of a two-point distribution is off by at most half a code's distance / sqrt(n), five times."""
    n = 1 << 16
    p = torch.zeros(n, device="cuda")
    g = torch.full((n,), 0.37, device="cuda")
    g[::256] = 1.0                                                   # the largest of every block
    for seed in range(3):
        m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        sm, sv = (torch.zeros(n // 256, device="cuda") for _ in range(2))
        binding.bagel_adamw_step([p], [g], [m], [v], 1, m_scale=[sm], v_scale=[sv], lr=0.0, weight_decay=0.0, seed=seed)
        keep = torch.arange(n) % 256 != 0
        for codes, scale, want in ((m, sm, 0.1 * 0.37), (v, sv, math.sqrt(0.001) * 0.37)):
            x = _values(codes, scale)[keep]
            distance = 16 * float(scale[0])                          # 0.37 * 448 = 165.8 lies between 160 and 176
            assert x.unique().numel() == 2
            assert abs(float(x.mean()) - want) <= 5 * distance / 2 / math.sqrt(n)
    # Over 4000 updates with gradients of 1 beside one of 3 in every block, sqrt(v) climbs to 1 from nothing, where a code is 6 to 12 % away
    # from the next and an update moves it by 0.05 % at most.  The same updates in plain form end within 2 % with a spread of 5 %
    # from place to place.
    n = 1 << 12
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    sm, sv = (torch.zeros(n // 256, device="cuda") for _ in range(2))
    p = torch.zeros(n, device="cuda")
    g = torch.ones(n, device="cuda")
    g[::256] = 3.0
    for t in range(1, 4001):
        binding.bagel_adamw_step([p], [g], [m], [v], t, m_scale=[sm], v_scale=[sv], lr=0.0, weight_decay=0.0, seed=9)
    root, want = _values(v, sv)[torch.arange(n) % 256 != 0], math.sqrt(1 - 0.999 ** 4000)
    assert abs(float(root.mean()) / want - 1) < 0.05 and float(root.std()) / want < 0.15


@gpu
def test_adamw_changes_nothing_where_the_scale_is_not_finite():
    for bad in (float("inf"), float("nan")):
        t = [_normal((300,), i).abs().cuda() for i in range(4)]
        before = [x.clone() for x in t]
        binding.bagel_adamw_step(*[[x] for x in t], 3, grad_scale=torch.tensor([bad], device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(t, before))


@gpu
def test_adamw_in_8_bits_of_zeros_and_tiny_blocks():
    n = 600
    p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    g[256:512] = 1e-38
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    sm, sv = (torch.zeros(3, device="cuda") for _ in range(2))
    for t in (1, 2, 3):
        binding.bagel_adamw_step([p], [g], [m], [v], t, m_scale=[sm], v_scale=[sv], weight_decay=0.0)
    assert torch.isfinite(p).all() and torch.isfinite(sm).all() and torch.isfinite(sv).all()
    assert not m.float().any() and bool((p[:256] == 1).all()) and bool((p[512:] == 1).all())


# ------------------------------------------------------------------------------------------------------ streams and graphs
def _all_calls(stream=None):
    """Every call once on small inputs; (launch, outputs)."""
    rows, width, at = 300, 136, [0, 130, 300]
    x = _cuda(_join_inputs(rows, width, torch.bfloat16, "silu"))
    rest = dict(act="silu", stream=stream, **{k: x[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
    out, normed, d_branch, d_value, d_forget, hidden = (torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda") for _ in range(6))
    d_scale, d_bias, bias = (torch.zeros(width, device="cuda") for _ in range(3))
    final, state = torch.zeros(2, width, device="cuda"), torch.zeros(rows, width, device="cuda")
    carry = torch.zeros(binding.bagel_recurrence_carry_rows(rows), width, device="cuda")
    offsets = torch.tensor(at, dtype=torch.int32).cuda()
    spaces = [torch.empty(k, dtype=torch.uint8, device="cuda")
              for k in (binding.bagel_block_join_workspace(rows, width), binding.bagel_recurrence_workspace(rows, width))]
    p, m, v = _normal((rows, width), 50).cuda(), torch.zeros(rows, width, device="cuda"), torch.zeros(rows, width, device="cuda")

    def launch():
        binding.bagel_block_join(x["branch"], x["resid"], out, normed, **rest)
        binding.bagel_recurrence(normed, x["gate"], hidden, offsets, bias=bias, final=final, carry=carry, workspace=spaces[1], stream=stream)
        binding.bagel_recurrence_grad(normed, x["gate"], hidden, d_value, d_forget, offsets, carry, bias=bias, d_bias=d_bias,
                                      workspace=spaces[1], stream=stream)
        binding.bagel_block_join_grad(x["branch"], out, d_value, d_forget, d_branch=d_branch, d_scale=d_scale, workspace=spaces[0], **rest)
        binding.bagel_recurrence_step(d_branch, x["gate"], state, bias=bias, stream=stream)
        binding.bagel_adamw_step([p], [d_branch], [m], [v], 3, stream=stream)

    outputs = [out, normed, hidden, final, d_value, d_forget, d_bias, d_branch, d_scale, state, p, m, v]
    return launch, outputs, x


@gpu
def test_another_stream():
    launch, want, _ = _all_calls()
    launch()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    launch, got, _ = _all_calls(side)
    side.wait_stream(torch.cuda.current_stream())
    launch()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@gpu
def test_in_a_graph():
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
        for name in ("branch", "resid", "gate"):
            new = _normal(x[name].shape, 100 * k + len(name), torch.bfloat16).cuda()
            x[name].copy_(new)
            y[name].copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        eager()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), k


# --------------------------------------------------------------------------------------------------------------- refusals
def _refused(call, args, text):
    lib = binding.load()
    assert getattr(lib, call)(C.byref(args), None) == binding.EINVAL
    message = lib.bagel_last_error(None).decode()
    assert message.startswith(call + ":") and text in message, message


def _join_struct(**kw):
    a = binding._Join()
    a.rows, a.width, a.dtype, a.act, a.eps = 4, 32, 0, 0, 1e-6
    for k in ("branch", "resid", "out", "normed"):
        setattr(a, k, 0x10000)
        setattr(a, k + "_stride", 32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,text", [
    (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(width=16385), "width"), (dict(dtype=3), "dtype"), (dict(act=4), "act"),
    (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(act=1), "gate"), (dict(gate=0x10000), "gate"), (dict(resid_stride=31), "stride"),
    (dict(resid=0x10002), "stride"), (dict(out=None, normed=None), "left out"), (dict(branch=None, resid=None), "left out")])
def test_join_refuses(change, text):
    _refused("bagel_block_join", _join_struct(**change), text)


@pytest.mark.parametrize("change,text", [
    (dict(out=None), "out"), (dict(d_scale=0x10000), "workspace"), (dict(d_scale=0x10000, workspace=0x10000, workspace_bytes=16), "too small"),
    (dict(d_scale=0x10000, workspace=0x10008, workspace_bytes=1 << 20), "16 bytes"), (dict(d_gate=0x10000, d_gate_stride=32), "d_gate"),
    (dict(branch=None, d_branch=0x10000, d_branch_stride=32), "branch"), (dict(d_out=0x10000, d_out_stride=4), "stride")])
def test_join_grad_refuses(change, text):
    _refused("bagel_block_join_grad", _join_struct(**change), text)


def _recurrence_struct(**kw):
    a = binding._Recurrence()
    a.rows, a.width, a.dtype, a.sequences = 6, 32, 1, 2
    for k in ("value", "forget", "hidden", "d_hidden"):
        setattr(a, k, 0x10000)
        setattr(a, k + "_stride", 32)
    a.carry = a.workspace = a.state = 0x10000
    a.workspace_bytes = 1 << 20
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("call", ["bagel_recurrence", "bagel_recurrence_grad"])
@pytest.mark.parametrize("change,text", [
    (dict(rows=-1), "rows"), (dict(rows=2 ** 31 - 1), "rows"), (dict(width=0), "width"), (dict(width=1 << 20), "width"), (dict(dtype=-1), "dtype"),
    (dict(sequences=-1), "sequences"), (dict(sequences=0), "sequence"), (dict(sequences=4), "divide"), (dict(value=None), "value"),
    (dict(forget=None), "forget"), (dict(workspace=None), "workspace"), (dict(workspace_bytes=8), "too small"), (dict(workspace=0x10004), "16 bytes"),
    (dict(value_stride=16), "stride"), (dict(forget=0x10001), "stride")])
def test_recurrence_refuses(call, change, text):
    _refused(call, _recurrence_struct(**change), text)


def test_recurrence_parts_are_needed():
    _refused("bagel_recurrence", _recurrence_struct(hidden=None), "hidden")
    _refused("bagel_recurrence_grad", _recurrence_struct(d_hidden=None), "d_hidden")
    _refused("bagel_recurrence_grad", _recurrence_struct(carry=None), "carry")
    _refused("bagel_recurrence_step", _recurrence_struct(state=None), "state")
    _refused("bagel_recurrence_step", _recurrence_struct(width=0), "width")
    lib = binding.load()
    assert lib.bagel_recurrence(None, None) == lib.bagel_block_join(None, None) == lib.bagel_recurrence_step(None, None) == binding.EINVAL
    assert lib.bagel_recurrence_carry_rows(-1) == lib.bagel_recurrence_workspace(5, 0) == lib.bagel_block_join_workspace(-1, 8) == binding.EINVAL
    assert lib.bagel_recurrence_carry_rows(0) == 0 and lib.bagel_recurrence_carry_rows(1) == 1 and lib.bagel_recurrence_carry_rows(129) == 2


@pytest.mark.parametrize("change,tensor,text", [
    (dict(step=0), {}, "step"), (dict(lr=-1.0), {}, "lr"), (dict(lr=float("inf")), {}, "lr"), (dict(beta1=1.0), {}, "betas"),
    (dict(beta2=-0.1), {}, "betas"), (dict(eps=0.0), {}, "eps"), (dict(eps=1e-60), {}, "eps"), (dict(grad_dtype=7), {}, "dtype"),
    (dict(state_bits=4), {}, "state_bits"), (dict(state_bits=8), {}, "m_scale"), ({}, dict(count=-1), "count"), ({}, dict(param=None), "null"),
    ({}, dict(m=0x10001), "multiple"), ({}, dict(grad=0x10002), "multiple"), ({}, dict(weight_decay=-1.0), "weight_decay"),
    ({}, dict(weight_decay=1e6), "weight_decay"), ({}, dict(weight_decay=float("nan")), "weight_decay")])
def test_adamw_refuses(change, tensor, text):
    o, t = binding._AdamW(), (binding._AdamWTensor * 1)()
    o.step, o.lr, o.beta1, o.beta2, o.eps, o.state_bits = 1, 1e-3, 0.9, 0.999, 1e-8, 32
    t[0].param = t[0].grad = t[0].m = t[0].v = 0x10000
    t[0].count = 5
    for k, v in change.items():
        setattr(o, k, v)
    for k, v in tensor.items():
        setattr(t[0], k, v)
    lib = binding.load()
    assert lib.bagel_adamw_step(t, 1, C.byref(o), None) == binding.EINVAL
    assert text in lib.bagel_last_error(None).decode()
    assert lib.bagel_adamw_step(None, 1, C.byref(o), None) == lib.bagel_adamw_step(t, -1, C.byref(o), None) == binding.EINVAL


def test_structures_are_those_of_the_header(tmp_path):
    """The binding's structures have the size and the places of the C header's."""
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
int main(void) { printf("%zu %zu %zu %zu %zu %zu %zu %d %d %d\\n", sizeof(bagel_join), sizeof(bagel_gated_recurrence), sizeof(bagel_adamw_tensor),
sizeof(bagel_adamw), offsetof(bagel_join, workspace), offsetof(bagel_gated_recurrence, workspace), offsetof(bagel_adamw, seed),
BAGEL_JOIN_MAX_WIDTH, BAGEL_RECURRENCE_SPAN, BAGEL_ADAMW_BLOCK); return 0; }""")
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", exe, str(src)], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    b = binding
    assert got == [C.sizeof(b._Join), C.sizeof(b._Recurrence), C.sizeof(b._AdamWTensor), C.sizeof(b._AdamW), b._Join.workspace.offset,
                   b._Recurrence.workspace.offset, b._AdamW.seed.offset, b.JOIN_MAX_WIDTH, b.RECURRENCE_SPAN, b.ADAMW_BLOCK]


def test_binding_refuses_before_the_library_is_called():
    x = torch.zeros(4, 8)
    for call in (lambda: binding.bagel_block_join(x, x, x), lambda: binding.bagel_recurrence(x, x, x, 1), lambda: binding.bagel_recurrence_step(x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="act"):
        binding.bagel_block_join(x, x, x, act="tanh")
    with pytest.raises(ValueError, match="lists"):
        binding.bagel_adamw_step([x], [], [x], [x], 1)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        binding.bagel_block_join(x.double(), x.double(), x.double())


@gpu
def test_binding_refuses_on_the_gpu():
    x = torch.zeros(4, 8, device="cuda")
    for bad in (x[:, :4], x.t().contiguous().t(), x.half(), x.cpu(), x[None], "text"):
        with pytest.raises(ValueError):
            binding.bagel_block_join(x, x, bad)
        with pytest.raises(ValueError):
            binding.bagel_recurrence(x, bad, x, 1)
    with pytest.raises(ValueError, match="offsets"):
        binding.bagel_recurrence(x, x, x, torch.tensor([0, 4], device="cuda"))
    with pytest.raises(binding.BagelError, match="divide"):
        binding.bagel_recurrence(x, x, x, 3)
    with pytest.raises(ValueError, match="workspace"):
        binding.bagel_recurrence(x, x, x, 1, workspace=x)
    with pytest.raises(binding.BagelError, match="too small"):
        binding.bagel_recurrence(x, x, torch.empty_like(x), 1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="tensor 0"):
        binding.bagel_adamw_step([x], [x[0]], [x], [x], 1)
