"""Edges of the operators of a policy with memory: gates that are nearly open or shut, large biases, infinities, draws of the moments in 8
bits, arguments that have to be refused, and sizes at which a workgroup goes through several rows or blocks.

Tolerances are those of test_operators.py where no other is derived."""
import concurrent.futures
import ctypes as C
import os
import shutil
import subprocess
import sys

import pytest
import torch

import test_operators as ops
from paper_2202_13638_amd import binding

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ULP = 2.0 ** -23


# ------------------------------------------------------------------------------------------------------ gated recurrence
@gpu
@pytest.mark.parametrize("size", [0.0, 50.0, 200.0, 1000.0])
def test_a_gate_of_a_large_bias_and_a_forget_gate_against_it(size):
    """q depends on forget + bias alone, whose sum is exact here.  With z that sum: 2^-24 of z from its product with log2(e), and 2^-25 from
    that constant, move the exponential by 1.1 |z| 2^-24; exponential, 1 + e, reciprocal, product and the new state round five times by a unit at
    most.  Held to twice that."""
    width, rows = 96, 40
    z, bias = 3 * ops._normal((rows, width), 1), size * torch.where(torch.arange(width) % 2 == 0, 1.0, -1.0)
    f = z - bias
    z = f.double() + bias.double()
    q = torch.sigmoid(-z)
    state, hidden = torch.zeros(rows, width, device="cuda"), torch.empty(rows, width, device="cuda")
    binding.bagel_recurrence_step(torch.ones(rows, width, device="cuda"), f.cuda(), state, hidden, bias=bias.cuda())
    bound = (2 * z.abs() + 10) * ULP * q
    assert bool(((state.double().cpu() - q).abs() <= bound).all())
    r = ops._run_recurrence(torch.ones(rows, width, device="cuda"), f.cuda(), list(range(rows + 1)), bias.cuda(), None,
                            torch.ones(rows, width, device="cuda"), None)
    for got, want in ((r["hidden"], q), (r["final"], q), (r["d_value"], q), (r["d_forget"], -q * torch.sigmoid(z))):
        assert bool(((got.double().cpu() - want).abs() <= 2 * (2 * z.abs() + 10) * ULP * want.abs()).all())


BIASES = [-30.0, -18.0, -14.0, -10.0, -5.0, 0.0, 5.0, 10.0]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [64, 72, 260])
def test_gradients_of_gates_that_are_nearly_open(width, dtype):
    """A channel whose gate takes the value whole, 1 - q down to e^-32, has gradients of that size, and each is right by its own size: an optimiser that divides
    by a gradient's own size sees nothing else.  The share of a gate carries (1.3 |z| + 3) units (see above), a gradient two of them; a state
    that some hundred rows move is off by some twenty units.  Held to 4 |z| + 40 units of what is largest in the channel."""
    t, at = ops.TYPES[dtype], [0, 140, 141, 400]
    x, f, dh = (ops._normal((400, width), i, t, scale) for i, scale in ((1, 1.0), (2, 0.5), (3, 1.0)))
    bias = torch.tensor([BIASES[c % len(BIASES)] for c in range(width)])
    h0, dl = ops._normal((3, width), 5), ops._normal((3, width), 6)
    want, terms = ops._recurrence_ref(x, f, at, bias, h0, dh, dl)
    got = ops._run_recurrence(x.cuda(), f.cuda(), at, bias.cuda(), h0.cuda(), dh.cuda(), dl.cuda())
    units = (4 * (f.double() + bias).abs().amax(0) + 40) * ULP
    for k in ("hidden", "final", "d_value", "d_forget", "d_initial", "d_bias"):
        g, w = got[k].double().cpu(), want[k]
        bound = units * (terms if k == "d_bias" else w.abs().amax(0)) + 1.01 * ops.HALF_ULP[got[k].dtype] * w.abs()
        off = (g - w).abs() / bound
        assert bool((off <= 1).all()), f"{k}: {float(off.max()):.3g} times the bound, channel of bias {bias[int(off.amax(0).argmax()) if off.dim() > 1 else int(off.argmax())]}"


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_channels_beside_an_open_gate_have_the_same_bits(dtype):
    """Waves without an open gate go through other loops than waves with one."""
    t, width, at = ops.TYPES[dtype], 200, [0, 300, 300, 900, 1500]
    x, f, dh = (ops._normal((at[-1], width), i, t, 0.5).cuda() for i in (1, 2, 3))
    bias, h0, dl = ops._normal((width,), 4, mean=6.0, scale=0.2).cuda(), ops._normal((4, width), 5).cuda(), ops._normal((4, width), 6).cuda()
    a = ops._run_recurrence(x, f, at, bias, h0, dh, dl)
    open_ones = torch.tensor([5, 131, 199], device="cuda")
    bias[open_ones] = -9.0
    b = ops._run_recurrence(x, f, at, bias, h0, dh, dl)
    rest = torch.ones(width, dtype=torch.bool, device="cuda")
    rest[open_ones] = False
    for k in a:
        assert torch.equal(a[k][..., rest], b[k][..., rest]), k


@gpu
def test_a_value_that_replaces_a_large_state():
    """A state of 1e4 gives way to a value of a thousandth: what is left is the value and (1 - q) of the state, each to a rounding and to what the gate carries."""
    width = 64
    x, f = 1e-3 * (1 + ops._normal((1, width), 1).abs()), ops._normal((1, width), 2, scale=0.5)
    bias, h0 = torch.full((width,), -18.0), 1e4 * (1 + ops._normal((1, width), 3).abs())
    z = f.double() + bias
    want = torch.sigmoid(-z) * x.double() + torch.sigmoid(z) * h0.double()
    state, hidden = h0.cuda(), torch.empty(1, width, device="cuda")
    binding.bagel_recurrence_step(x.cuda(), f.cuda(), state, bias=bias.cuda())
    binding.bagel_recurrence(x.cuda(), f.cuda(), hidden, 1, bias=bias.cuda(), initial=h0.cuda())
    for got in (state, hidden):
        assert bool(((got.double().cpu() - want).abs() <= (4 * z.abs() + 40) * ULP * want).all())


def test_states_that_are_read_and_written_may_not_overlap():
    """Waves read the states before a sequence while others write those behind it."""
    for change in (dict(initial=0x20000, final=0x20000), dict(initial=0x20000, final=0x20000 + 4 * 63),
                   dict(initial=0x20000 + 4 * 63, final=0x20000)):
        ops._refused("bagel_recurrence", ops._recurrence_struct(rows=6, sequences=2, **change), "overlap")
    for change in (dict(d_final=0x20000, d_initial=0x20000), dict(d_final=0x20000, d_initial=0x20000 + 4 * 63)):
        ops._refused("bagel_recurrence_grad", ops._recurrence_struct(rows=6, sequences=2, **change), "overlap")


# ------------------------------------------------------------------------------------------------------------- block join
@gpu
@pytest.mark.parametrize("dtype", ops.TYPES)
@pytest.mark.parametrize("width", [8, 64, 320, 777, 2600, 16384])
def test_a_gate_that_is_shut_for_good(width, dtype):
    """A gate of minus infinity takes its entry of the branch out: silu and logistic are 0 there, and so are their derivatives."""
    t, rows = ops.TYPES[dtype], 5
    for act in ("silu", "logistic"):
        x = ops._join_inputs(rows, width, t, act)
        shut = torch.rand(rows, width, generator=torch.Generator().manual_seed(9)) < 0.3
        shut[3] = True                                              # a row of which nothing is left
        far = torch.where(shut, torch.tensor(-1e4), x["gate"].float()).to(t)
        x["gate"] = torch.where(shut, torch.tensor(float("-inf")), x["gate"].float()).to(t)
        g = _cuda(x)
        out, normed = torch.empty_like(g["resid"]), torch.empty_like(g["resid"])
        rest = dict(act=act, **{k: g[k] for k in ("gate", "post_weight", "scale", "pre_weight")})
        binding.bagel_block_join(g["branch"], g["resid"], out, normed, **rest)
        assert torch.equal(out.cpu()[shut], x["resid"][shut])
        # the reference has no infinite gates: at -1e4 its logistic function is exp(-1e4) = 0 in 64 bits too
        want = ops._join_ref(x["branch"], x["resid"], far, act, x["post_weight"], x["scale"], x["pre_weight"], 1e-6)
        ops._near(out, want[0], "out")
        ops._near(normed, want[1], "normed")
        got = ops._join_grad_case({**x, "gate": far}, g, out, ops._normal((rows, width), 7, t), ops._normal((rows, width), 8, t), act, 1e-6)
        assert not got["d_gate"].cpu()[shut].any()


def _cuda(d):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


def _close(got, want, name, terms=None):
    """_near of test_operators.py, where the tensors are."""
    w = want.double()
    bound = ops.HALF_ULP[got.dtype] * w.abs() * 1.01 + ops.WORK * (w.abs().max() if terms is None else terms)
    if got.dtype == torch.float16:
        bound = bound + 2.0 ** -25
    off = (got.double() - w).abs()
    assert bool((off <= bound).all()), f"{name}: off by {float(off.max()):.3g}, at most {float((off - bound).max()):.3g} too much"


# a width of every tile, in 32 bits; in 16 twice these (less one) fill the same tiles
TILES = [3, 101, 253, 511, 777, 1021, 1277, 1301, 1533, 2045, 2056, 3001, 4093, 5001, 8192, 12001]


@gpu
@pytest.mark.parametrize("dtype", ops.TYPES)
@pytest.mark.parametrize("width", TILES)
def test_join_of_more_rows_than_there_are_places(width, dtype):
    """Every tile with several rows to a workgroup: forward there are at most 4096 workgroups, back 512 or 1024, of one row or of four."""
    t = ops.TYPES[dtype]
    width = width if dtype == "f32" or width > 8192 else 2 * width - (width % 8 != 0)
    packs = -(-width * t.itemsize // 16)
    forward, back = (20011, 5003) if packs <= 128 else (4211, 1301)
    act = ["silu", "logistic", "identity", "none"][(width + len(dtype)) % 4]
    g = torch.Generator(device="cuda").manual_seed(width)

    def normal(*shape, scale=1.0, mean=0.0, to=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * scale + mean).to(to)

    x = dict(branch=normal(forward, width, scale=0.7, to=t), resid=normal(forward, width, scale=2.0, to=t),
             gate=normal(forward, width, scale=1.5, to=t) if act != "none" else None, post_weight=normal(width, scale=0.2, mean=1.0),
             scale=normal(width, scale=0.2, mean=0.3), pre_weight=normal(width, scale=0.2, mean=1.0))
    vectors = {k: x[k] for k in ("post_weight", "scale", "pre_weight")}
    out, normed = (torch.full((forward, width), float("nan"), dtype=t, device="cuda") for _ in range(2))
    binding.bagel_block_join(x["branch"], x["resid"], out, normed, gate=x["gate"], act=act, eps=1e-5, **vectors)
    w, c, u = (v.double() for v in vectors.values())

    def norm(z):
        return torch.rsqrt(z.square().mean(1, keepdim=True) + 1e-5)

    z = x["branch"].double()
    a, _ = ops._act(x["gate"].double() if act != "none" else None, act)
    want = x["resid"].double() + c * w * z * norm(z) * (1.0 if a is None else a)
    _close(out, want, "out")
    _close(normed, want * norm(want) * u, "normed")
    del normed, want, z, a
    # back, by the formulas at the stored `out`; d_resid takes the place of d_out
    x = {k: v[:back] if v is not None and v.dim() == 2 else v for k, v in x.items()}
    out = out[:back]
    d_out, d_normed = normal(back, width, to=t), normal(back, width, to=t)
    o, z, dy, ro = out.double(), x["branch"].double(), d_normed.double(), norm(out.double())
    a, da = ops._act(x["gate"].double() if act != "none" else None, act)
    a, da = (torch.ones_like(z), torch.zeros_like(z)) if a is None else (a, da)
    n_out, rz = o * ro, norm(z)
    n = z * rz
    d = ro * (dy * u - n_out * (dy * u * n_out).mean(1, keepdim=True))
    dx = d_out.double() + d
    k = dx * c * w * a
    parts = d_out.double().abs() + d.abs() + 2 * (dy * u * ro).abs()
    want = {"d_resid": dx, "d_branch": rz * (k - n * (k * n).mean(1, keepdim=True)), "d_post_weight": (dx * c * a * n).sum(0), "d_scale": (dx * w * a * n).sum(0),
            "d_pre_weight": (dy * n_out).sum(0)}
    terms = {"d_resid": parts.max(), "d_branch": 2 * (parts * c * w * a * rz).abs().max(), "d_post_weight": (parts * c * a * n).abs().sum(0),
             "d_scale": (parts * w * a * n).abs().sum(0), "d_pre_weight": (dy * n_out).abs().sum(0)}
    if act != "none":
        want["d_gate"], terms["d_gate"] = dx * c * w * n * da, (parts * c * w * n * da).abs().max()
    got = {k: torch.full(v.shape, float("nan"), dtype=t if v.dim() == 2 else torch.float32, device="cuda") for k, v in want.items()}
    got["d_resid"] = d_out
    binding.bagel_block_join_grad(x["branch"], out, d_out, d_normed, gate=x["gate"], act=act, eps=1e-5, **vectors, **got)
    for k, v in want.items():
        _close(got[k], v, k, terms[k])


# ------------------------------------------------------------------------------------------------------------------ AdamW
def _draws(step, n=1 << 14, tensors=2, **kw):
    """For every place of some tensors of the same values whether its code was rounded up; the chance of that is (0.37 * 448 - 160) / 16 = 0.36."""
    grads = [torch.full((n,), 0.37, device="cuda") for _ in range(tensors)]
    for g in grads:
        g[::256] = 1.0                                               # the largest of every block
    p, m, v = ([torch.zeros(n, device="cuda").to(kind) for _ in range(tensors)] for kind in (torch.float32, torch.float8_e4m3fn, torch.float8_e4m3fn))
    sm, sv = ([torch.zeros(n // 256, device="cuda") for _ in range(tensors)] for _ in range(2))
    binding.bagel_adamw_step(p, grads, m, v, step, m_scale=sm, v_scale=sv, lr=0.0, weight_decay=0.0, **kw)
    codes = torch.stack([c.float() for c in m])
    here = torch.arange(n, device="cuda") % 256 != 0
    assert set(codes[:, here].unique().tolist()) == {160.0, 176.0}
    return (codes == 176).float(), here


def _independent(a, b, here):
    """Draws that have nothing to do with each other agree in 0.36^2 + 0.64^2 of all places, within five standard deviations."""
    same = 0.36 ** 2 + 0.64 ** 2
    return abs(float((a == b)[here].float().mean()) - same) < 5 * (same * (1 - same) / int(here.sum())) ** 0.5


@gpu
def test_draws_of_neighbours_updates_and_tensors_are_independent():
    (a, here), (b, _), (again, _), (other, _) = _draws(41), _draws(42), _draws(41), _draws(41, run=1)
    assert torch.equal(a, again)                                     # equal calls give equal results
    for shift in (0, 1, 2, 17):                                      # the next update is not this one moved on
        both = here & here.roll(-shift)
        assert _independent(a.roll(-shift, 1)[0], b[0], both), shift
        assert shift == 0 or _independent(a.roll(-shift, 1)[0], a[0], both), shift
    assert _independent(a[0], a[1], here)                            # two tensors of one update
    assert _independent(a[0], other[0], here)                        # and of two calls with other numbers


@gpu
def test_roots_of_a_long_run_scatter_from_place_to_place_only():
    """sqrt(v) climbs from nothing over 4000 updates with gradients of 1 beside one of 3 in every block.  From place to place its codes scatter by 5 % (see
    test_adamw_in_8_bits_keeps_means); where the draws are independent the mean of a block's 255 scatters by 0.05 / sqrt(255) = 0.3 %.  Held to 1 %."""
    n = 1 << 13
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    sm, sv = (torch.zeros(n // 256, device="cuda") for _ in range(2))
    p, g = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    g[::256] = 3.0
    for t in range(1, 4001):
        binding.bagel_adamw_step([p], [g], [m], [v], t, m_scale=[sm], v_scale=[sv], lr=0.0, weight_decay=0.0)
    root = ops._values(v, sv).view(-1, 256)[:, 1:]
    want = (1 - 0.999 ** 4000) ** 0.5
    assert abs(float(root.mean()) / want - 1) < 0.01
    assert float(root.mean(1).std()) / want < 0.01


@gpu
@pytest.mark.parametrize("step,seed", [(1, 0), (42, 7), (1 << 20, 0xFFFFFFFF)])
def test_draws_of_a_given_number_are_those_that_are_documented(step, seed):
    mask = 0xFFFFFFFF
    got, here = _draws(step, seed=seed)
    x = (torch.arange(got.shape[1]) * 0x9E3779B9 + seed * 0xBB67AE85 + step * 0x9E3779B9) & mask
    x = ((x ^ (x >> 16)) * 0x6A09E667) & mask
    x = ((x ^ (x >> 15)) * 0x3C6EF373) & mask
    low = ((x ^ (x >> 16)) & 0xFFFF)[here.cpu()]
    sure = ((low.double() / 65536 - 0.64).abs() > 1e-4)              # 0.37 * 448 itself is rounded
    for tensor in got.cpu():
        assert torch.equal((tensor[here.cpu()] == 1)[sure], (low >= 0.64 * 65536)[sure])


@gpu
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 1e30])
def test_an_infinity_takes_its_own_place_of_a_block_in_8_bits(bad):
    """As in 32 bits: what is not finite is kept as that, and the other 255 of its block go on as if a small number stood there."""
    n, at = 700, 300

    def run(first):
        p, g = ops._normal((n,), 1).cuda(), ops._normal((n,), 2).cuda()
        m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        sm, sv = (torch.zeros(3, device="cuda") for _ in range(2))
        for t in range(1, 5):
            g = ops._normal((n,), 2 + t).cuda()
            g[at] = first if t == 2 else 1e-3
            binding.bagel_adamw_step([p], [g], [m], [v], t, m_scale=[sm], v_scale=[sv], seed=t)
        return p, m, v, sm, sv

    want, got = run(1e-3), run(bad)
    rest = torch.arange(n, device="cuda") != at
    assert torch.equal(want[4], got[4]) and torch.equal(want[2].view(torch.uint8)[rest], got[2].view(torch.uint8)[rest])
    assert torch.isnan(got[0][at])                                   # v is infinite, its step is no number
    if abs(bad) == 1e30:
        assert all(torch.isfinite(t.float()[rest]).all() for t in (got[0], got[1]))       # m is finite, and the largest of its block
    else:
        assert torch.equal(want[0][rest], got[0][rest]) and torch.equal(want[3], got[3])
        assert torch.equal(want[1].view(torch.uint8)[rest], got[1].view(torch.uint8)[rest])


@gpu
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_adamw_in_8_bits_of_four_blocks_a_wave(grad):
    """From 16384 blocks on a wave takes four of them one after the other; the last block of the last is not whole."""
    ops.test_adamw_in_8_bits((4_300_007,), grad)


# --------------------------------------------------------------------------------------------- arguments, streams, errors
def test_lists_of_an_update_are_lists():
    """What is given and is no list of as many entries is refused, and so are scales beside moments in 32 bits: none is left out in silence."""
    x = torch.zeros(4)
    for bad in (5, True, object()):
        with pytest.raises(ValueError, match="copy"):
            binding.bagel_adamw_step([x], [x], [x], [x], 1, copy=bad)
    with pytest.raises(ValueError, match="lists"):
        binding.bagel_adamw_step([x], [x], [x], [x], 1, copy=[x, x])
    for name in ("m_scale", "v_scale"):
        for bad in ([x], 5, [x, x]):
            with pytest.raises(ValueError, match=name):
                binding.bagel_adamw_step([x], [x], [x], [x], 1, **{name: bad})


@gpu
def test_lists_of_an_update_are_lists_on_the_gpu():
    x = [torch.zeros(4, device="cuda") for _ in range(5)]
    with pytest.raises(ValueError, match="copy"):
        binding.bagel_adamw_step([x[0]], [x[1]], [x[2]], [x[3]], 1, copy=5)
    with pytest.raises(ValueError, match="m_scale"):
        binding.bagel_adamw_step([x[0]], [x[1]], [x[2]], [x[3]], 1, m_scale=[x[4]], v_scale=[x[4]])
    binding.bagel_adamw_step([x[0]], [x[1]], [x[2]], [x[3]], 1, m_scale=[None], v_scale=[None])       # nothing is there


@gpu
def test_numbers_that_do_not_fit_are_refused():
    x = torch.zeros(4, 8, device="cuda")
    for offsets in (2 ** 31, 2 ** 40, 2 ** 70, -2 ** 40, "two", None):
        with pytest.raises(ValueError, match="offsets"):
            binding.bagel_recurrence(x, x, torch.empty_like(x), offsets)
    with pytest.raises(ValueError, match="eps"):
        binding.bagel_block_join(x, x, torch.empty_like(x), eps="small")
    with pytest.raises(binding.BagelError, match="eps"):             # infinite in 32 bits
        binding.bagel_block_join(x, x, torch.empty_like(x), eps=1e60)
    for kw in (dict(step=2 ** 70), dict(step="one"), dict(lr="fast"), dict(beta1=None), dict(seed=object()), dict(run="a")):
        with pytest.raises(ValueError, match=next(iter(kw))):
            binding.bagel_adamw_step(*[[torch.zeros(4, device="cuda")] for _ in range(4)], **{"step": 1, **kw})
    # sizes beyond the library's, where a work space is to be made first: the library's own refusal
    wide, vector = torch.zeros(1, 16400, device="cuda"), torch.zeros(16400, device="cuda")
    with pytest.raises(binding.BagelError, match="width"):
        binding.bagel_block_join_grad(wide, wide, wide, d_scale=vector)
    wide = torch.zeros(1, 1 << 20, device="cuda")
    with pytest.raises(binding.BagelError, match="width"):
        binding.bagel_recurrence(wide, wide, torch.empty_like(wide), 1)


def test_the_message_of_a_failed_call_stays():
    lib = binding.load()
    ctx = C.c_void_p()
    assert lib.bagel_create(C.byref(ctx), None, None) == binding.EINVAL
    message = lib.bagel_last_error(None)
    assert message.startswith(b"bagel_create:")
    o = binding._AdamW()
    o.step, o.lr, o.eps, o.state_bits = 1, 1e-3, 1e-8, 32
    assert lib.bagel_adamw_step(None, 0, C.byref(o), None) == binding.OK          # no tensors: nothing to do
    assert lib.bagel_last_error(None) == message


@gpu
def test_work_spaces_on_another_stream():
    """Without one of the caller's, a call on another stream makes its work space there."""
    rows, width = 3000, 264
    x, f, dh = (ops._normal((rows, width), i, torch.bfloat16).cuda() for i in (1, 2, 3))
    j = _cuda(ops._join_inputs(rows, width, torch.bfloat16, "silu"))
    rest = dict(act="silu", **{k: j[k] for k in ("gate", "post_weight", "scale", "pre_weight")})

    def calls(stream):
        r = [torch.zeros_like(x) for _ in range(4)]
        vectors = {k: torch.zeros(width, device="cuda") for k in ("d_post_weight", "d_scale", "d_pre_weight")}
        d_bias, carry = torch.zeros(width, device="cuda"), torch.zeros(binding.bagel_recurrence_carry_rows(rows), width, device="cuda")
        torch.cuda.synchronize()
        for _ in range(3):
            binding.bagel_recurrence(x, f, r[0], 1, carry=carry, stream=stream)
            binding.bagel_recurrence_grad(x, f, dh, r[1], r[2], 1, carry, d_bias=d_bias, stream=stream)
            binding.bagel_block_join_grad(j["branch"], j["resid"], x, dh, d_branch=r[3], stream=stream, **vectors, **rest)
        torch.cuda.synchronize()
        return [*r, d_bias, *vectors.values()]

    assert all(torch.equal(a, b) for a, b in zip(calls(None), calls(torch.cuda.Stream())))


def test_first_calls_from_several_threads():
    """The library is looked up by whoever comes first; nobody sees half of it."""
    code = ("import threading, torch\nfrom paper_2202_13638_amd import binding\nx, got = torch.zeros(2, 2), []\nstart = threading.Barrier(8)\n"
            "def call():\n    start.wait()\n    try:\n        binding.bagel_block_join(x, x, x)\n    except Exception as e:\n        got.append(type(e).__name__)\n"
            "t = [threading.Thread(target=call) for _ in range(8)]\n[i.start() for i in t]\n[i.join() for i in t]\nprint(got)\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith(str(["ValueError"] * 8)), r.stdout + r.stderr


@pytest.mark.slow
def test_host_side_of_the_operators_under_sanitizers(tmp_path):
    """AddressSanitizer and UndefinedBehaviorSanitizer on host code; device code as the library has it.  No GPU is involved."""
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not found")
    from paper_2202_13638_amd import build
    build.build()
    units = ["adamw.hip", "bagel_api.hip", "block_join.hip", "recurrence.hip"]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    sources = [os.path.join(build.CSRC, u) for u in units] + [os.path.join(ROOT, "tests", "sanitize", "operators_driver.cpp")]

    def compiled(source):
        obj = str(tmp_path / (os.path.basename(source) + ".o"))
        r = subprocess.run(["hipcc", *build.FLAGS, "-g", "-x", "hip", *san, "-c", source, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return obj

    with concurrent.futures.ThreadPoolExecutor(len(sources)) as pool:
        objs = list(pool.map(compiled, sources))
    objs += [os.path.join(build.BUILD, s.replace(".hip", ".o")) for s in build.SOURCES if s not in units]
    exe = str(tmp_path / "operators_san")
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", "-o", exe, *objs],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    # the HIP runtime keeps allocations of its own to the end
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "operators sanitizer driver: ok" in out, out
    assert "ERROR: AddressSanitizer" not in out and "runtime error" not in out, out
