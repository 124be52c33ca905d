"""The operators of a policy with memory, as they are measured: what they compute in plain form, and the calls that compute it.

A policy with memory is a stack of recurrent blocks over the steps of recorded trajectories.  A case is one call (or one
forward and backward pass) of one operator, by `kind`:

  join        the end of one block and the start of the next.  With R(z) = z / sqrt(mean(z^2) + eps) over a row,
                out = resid + scale * act(gate) * (R(branch) * post_weight),   normed = R(out) * pre_weight;
              act is the identity, the logistic function or z * logistic(z)
  join_grad   its gradient with respect to every input, at the `out` that was stored
  recurrence  the gated linear recurrence of every channel along a sequence, q_t = logistic(-(forget_t + bias)),
                h_t = (1 - q_t) h_{t-1} + q_t value_t,
              over sequences of different lengths packed one after the other, and its gradient
  step        one step of it for many sequences at once, the state updated in place
  adamw       an update of many tensors at once, the moments in 32 bits, or in 8 with a scale for every 256 values

Moments in 8 bits are float8_e4m3fn codes times their block's scale = largest / 448.  The second moment is held as its square
root.  A code is rounded up or down by chance, in proportion to its distance from both; the random bits are a hash of the place in
the tensor, the number of the update and a seed.  A root that is not zero never gets the code of zero.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256                  # values of a moment in 8 bits that share a scale
LARGEST = 448.0              # largest value of float8_e4m3fn
KINDS = ("join", "join_grad", "recurrence", "step", "adamw")


def listed():
    return [
        # a controller serving a few machines: one row each, so latency is all there is
        {"name": "join_serve", "kind": "join", "rows": 16, "width": 512, "dtype": "bf16", "act": "silu"},
        # the recorded trajectories of a training batch: 64 of 1000 steps
        {"name": "join_batch", "kind": "join", "rows": 64000, "width": 1024, "dtype": "bf16", "act": "silu"},
        # the backward pass of a large batch through a wide block
        {"name": "join_grad_large", "kind": "join_grad", "rows": 65536, "width": 4096, "dtype": "bf16", "act": "silu"},
        # a width that fits no vector and no tile, in 32 bits
        {"name": "join_grad_odd", "kind": "join_grad", "rows": 9973, "width": 777, "dtype": "f32", "act": "logistic"},
        # one control period of 256 machines
        {"name": "step_serve", "kind": "step", "sequences": 256, "width": 512, "dtype": "bf16"},
        # a training batch in 32 bits: 64 trajectories of 1000 steps
        {"name": "recurrence_batch", "kind": "recurrence", "tokens": 64000, "sequences": 64, "lengths": "equal", "width": 512,
         "dtype": "f32"},
        # one very long recording: the only work to share out lies along it
        {"name": "recurrence_long", "kind": "recurrence", "tokens": 131072, "sequences": 1, "lengths": "equal", "width": 1024,
         "dtype": "bf16"},
        # episodes that ended at different times, some at once, packed one after the other; an odd width
        {"name": "recurrence_packed", "kind": "recurrence", "tokens": 50021, "sequences": 61, "lengths": "ragged", "width": 777,
         "dtype": "f16"},
        # the largest memoryless policy: six tensors of 1 to 65536 values
        {"name": "adamw_policy", "kind": "adamw", "sizes": "256x5,256,256x256,256,256,1", "repeat": 1, "bits": 32, "grad": "f32",
         "copy": "none"},
        # a policy of eight blocks, 64 tensors; gradients and working weights in bf16
        {"name": "adamw_blocks", "kind": "adamw", "sizes": "1024x1024,1024x1024,1024x1024,1024x1024,1024,1024,1024,1024", "repeat": 8,
         "bits": 32, "grad": "bf16", "copy": "bf16"},
        # a large model whose moments only fit in 8 bits
        {"name": "adamw_large_8bit", "kind": "adamw", "sizes": "4096x4096,4096x4096,4096x4096,4096x4096,4096,4096,4096,4096", "repeat": 6,
         "bits": 8, "grad": "bf16", "copy": "bf16"},
        # tensors that end inside a block of 256, some of one or two values
        {"name": "adamw_odd_8bit", "kind": "adamw", "sizes": "777x333,777,1,255,257,333x777,64009,2", "repeat": 5, "bits": 8, "grad": "f32",
         "copy": "none"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(KINDS)
    dtype = rng.choice(sorted(DTYPES))
    if kind in ("join", "join_grad"):
        width = _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            width = 2 ** round(math.log2(width))
        rows = _log_int(rng, 1, 65536 * 4096 // (width * (2 if dtype == "f32" else 1)))
        return {"kind": kind, "rows": min(rows, 262144), "width": width, "dtype": dtype, "act": rng.choice(["none", "identity", "logistic", "silu"])}
    if kind == "step":
        return {"kind": kind, "sequences": _log_int(rng, 1, 4096), "width": _log_int(rng, 16, 4096), "dtype": dtype}
    if kind == "recurrence":
        width = _log_int(rng, 16, 2048)
        if rng.random() < 0.5:
            width = 2 ** round(math.log2(width))
        tokens = _log_int(rng, 64, min(131072, 131072 * 1024 // (width * (2 if dtype == "f32" else 1))))
        lengths = rng.choice(["equal", "ragged"])
        sequences = _log_int(rng, 1, max(1, min(512, tokens // 16)))
        if lengths == "equal":
            tokens = max(1, tokens // sequences) * sequences
        return {"kind": kind, "tokens": tokens, "sequences": sequences, "lengths": lengths, "width": width, "dtype": dtype}
    repeat = _log_int(rng, 1, 24)
    total = _log_int(rng, 2000, 4e8) // repeat
    sizes, count = [], rng.randint(1, 8)
    for _ in range(count):
        n = _log_int(rng, 1, max(1, total // count))
        if n > 4096 and rng.random() < 0.5:
            side = _log_int(rng, 16, n // 16)
            sizes.append("%dx%d" % (side, n // side))
        else:
            sizes.append(str(n))
    return {"kind": kind, "sizes": ",".join(sizes), "repeat": repeat, "bits": rng.choice([8, 32]), "grad": dtype,
            "copy": rng.choice(["none", "bf16", "f16"])}


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["sizes"].split(",")] * case["repeat"]


def _offsets(case, g):
    """Where the sequences begin, and where the last one ends: lengths spread about their mean, one in eight of them zero."""
    n, tokens = case["sequences"], case["tokens"]
    if case["lengths"] == "equal":
        return [i * (tokens // n) for i in range(n + 1)]
    w = torch.rand(n, generator=g).square() + 0.01
    w[torch.rand(n, generator=g) < 0.125] = 0
    w[torch.randint(n, (1,), generator=g)] += 0.5
    ends = (torch.cumsum(w.double(), 0) / w.double().sum() * tokens).round().long().tolist()
    return [0] + ends[:-1] + [tokens]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]

    def normal(*shape, scale=1.0, mean=0.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(mean).to(dtype)

    s = {"case": dict(case)}
    if kind in ("join", "join_grad"):
        r, d, t = case["rows"], case["width"], DTYPES[case["dtype"]]
        s["branch"] = normal(r, d, scale=0.7, dtype=t)
        s["gate"] = normal(r, d, dtype=t) if case["act"] != "none" else None
        s["resid" if kind == "join" else "out"] = normal(r, d, scale=2.0, dtype=t)
        s["post_weight"], s["pre_weight"] = normal(d, scale=0.1, mean=1.0), normal(d, scale=0.1, mean=1.0)
        s["scale"] = normal(d, scale=0.05, mean=0.2)
        if kind == "join_grad":
            s["d_out"], s["d_normed"] = normal(r, d, scale=1e-2, dtype=t), normal(r, d, scale=1e-2, dtype=t)
    elif kind == "step":
        n, d, t = case["sequences"], case["width"], DTYPES[case["dtype"]]
        s["value"], s["forget"] = normal(n, d, dtype=t), normal(n, d, dtype=t)
        s["bias"], s["state"] = normal(d, mean=3.0), normal(n, d, scale=0.3)
    elif kind == "recurrence":
        n, d, t = case["tokens"], case["width"], DTYPES[case["dtype"]]
        s["value"], s["forget"] = normal(n, d, dtype=t), normal(n, d, dtype=t)
        s["d_hidden"] = normal(n, d, scale=1e-2, dtype=t)
        s["bias"] = normal(d, mean=3.0)                       # memories of ten to a few hundred steps
        s["initial"], s["d_final"] = (normal(case["sequences"], d, scale=c) for c in (0.3, 1e-2))
        at = _offsets(case, torch.Generator().manual_seed(seed))
        s["offsets"] = torch.tensor(at, dtype=torch.int32, device="cuda")
    else:
        # Each kind of tensor in one allocation, as a trainer holds them, every tensor at a multiple of BLOCK values in it.
        shapes, total, places = _shapes(case), 0, []
        for shape in shapes:
            places.append((total, shape))
            total += -(-math.prod(shape) // BLOCK) * BLOCK

        def views(flat, each=1):
            return [flat[at // each: at // each + -(-math.prod(sh) // each)].view(sh if each == 1 else (-1,)) for at, sh in places]

        flat = {"p": normal(total, scale=0.1)}
        s["g"] = [normal(*sh, scale=1e-2, dtype=DTYPES[case["grad"]]) for sh in shapes]
        s["grad_scale"] = torch.full((1,), 0.37, device="cuda")
        s["update"], s["seed"] = 120, seed % 1000
        if case["copy"] != "none":
            flat["copy"] = torch.zeros(total, dtype=DTYPES[case["copy"]], device="cuda")
        if case["bits"] == 32:
            flat["m"], flat["v"] = normal(total, scale=1e-3), normal(total, scale=1e-3).square_().add_(1e-9)
        else:
            flat["m"] = normal(total, scale=100.0).clamp_(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
            flat["v"] = normal(total, scale=100.0).abs_().add_(2.0).clamp_(max=LARGEST).to(torch.float8_e4m3fn)
            for k in ("m_scale", "v_scale"):
                flat[k] = torch.rand(total // BLOCK, generator=g, device="cuda").mul_(1e-5).add_(1e-6)
        s["flat"] = flat
        for k in ("p", "m", "v", "copy", "m_scale", "v_scale"):
            s[k] = views(flat[k], BLOCK if k.endswith("scale") else 1) if k in flat else None
    return s


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2, "none": 0}
    kind = case["kind"]
    if kind in ("join", "join_grad"):
        n, e, gate = case["rows"] * case["width"], size[case["dtype"]], case["act"] != "none"
        if kind == "join":
            return {"bytes": n * e * (4 + gate) + 12 * case["width"], "flops": n * (9 + 4 * gate)}
        return {"bytes": n * e * (6 + 2 * gate) + 24 * case["width"], "flops": n * (22 + 10 * gate)}
    if kind == "step":
        n = case["sequences"] * case["width"]
        return {"bytes": n * (3 * size[case["dtype"]] + 8) + 4 * case["width"], "flops": 8 * n}
    if kind == "recurrence":
        n = case["tokens"] * case["width"]
        return {"bytes": n * 6 * size[case["dtype"]] + (16 * case["sequences"] + 8) * case["width"], "flops": 20 * n}
    n = sum(math.prod(sh) for sh in _shapes(case))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + state + size[case["grad"]] + size[case["copy"]]), "flops": n * (16 if case["bits"] == 32 else 60)}


# ------------------------------------------------------------------------------------------------ the calls, and the plain forms
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"join": _join_own, "join_grad": _join_grad_own, "step": _step_own, "recurrence": _recurrence_own, "adamw": _adamw_own}[kind](s)
    return {"join": _join_plain, "join_grad": _join_grad_plain, "step": _step_plain, "recurrence": _recurrence_plain, "adamw": _adamw_plain}[kind](s)


def _join_own(s):
    from paper_2202_13638_amd import binding
    out, normed = torch.empty_like(s["resid"]), torch.empty_like(s["resid"])
    binding.bagel_block_join(s["branch"], s["resid"], out, normed, gate=s["gate"], act=s["case"]["act"], post_weight=s["post_weight"],
                             scale=s["scale"], pre_weight=s["pre_weight"], eps=EPS)
    return {"out": out, "normed": normed}


def _join_grad_own(s):
    from paper_2202_13638_amd import binding
    like = torch.empty_like
    r = {"d_branch": like(s["branch"]), "d_resid": like(s["out"]), "d_gate": like(s["gate"]) if s["gate"] is not None else None,
         "d_post_weight": like(s["post_weight"]), "d_scale": like(s["scale"]), "d_pre_weight": like(s["pre_weight"])}
    binding.bagel_block_join_grad(s["branch"], s["out"], s["d_out"], s["d_normed"], gate=s["gate"], act=s["case"]["act"],
                                  post_weight=s["post_weight"], scale=s["scale"], pre_weight=s["pre_weight"], eps=EPS, **r)
    return r


def _step_own(s):
    from paper_2202_13638_amd import binding
    hidden = torch.empty_like(s["value"])
    binding.bagel_recurrence_step(s["value"], s["forget"], s["state"], hidden, bias=s["bias"])
    return {"hidden": hidden, "state": s["state"]}


def _recurrence_own(s):
    from paper_2202_13638_amd import binding
    like, (tokens, width) = torch.empty_like, s["value"].shape
    carry = torch.empty(binding.bagel_recurrence_carry_rows(tokens), width, device="cuda")
    r = {"hidden": like(s["value"]), "final": like(s["initial"]), "d_value": like(s["value"]), "d_forget": like(s["value"]),
         "d_initial": like(s["initial"]), "d_bias": like(s["bias"])}
    binding.bagel_recurrence(s["value"], s["forget"], r["hidden"], s["offsets"], bias=s["bias"], initial=s["initial"], final=r["final"],
                             carry=carry)
    binding.bagel_recurrence_grad(s["value"], s["forget"], s["d_hidden"], r["d_value"], r["d_forget"], s["offsets"], carry, bias=s["bias"],
                                  initial=s["initial"], d_final=s["d_final"], d_initial=r["d_initial"], d_bias=r["d_bias"])
    return r


def _adamw_own(s):
    from paper_2202_13638_amd import binding
    binding.bagel_adamw_step(s["p"], s["g"], s["m"], s["v"], s["update"], m_scale=s["m_scale"], v_scale=s["v_scale"], copy=s["copy"], lr=LR,
                             beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY, grad_scale=s["grad_scale"], seed=s["seed"])
    return s["flat"]                                          # the tensors' own memory


def _act(gate, act):
    """act(gate) and its derivative."""
    if act == "none":
        return 1.0, None
    if act == "identity":
        return gate, 1.0
    sig = 1 / (1 + torch.exp(-gate))
    if act == "logistic":
        return sig, sig * (1 - sig)
    return gate * sig, sig * (1 + gate * (1 - sig))


def _rms(z, eps=EPS):
    return torch.rsqrt((z * z).mean(-1, keepdim=True) + eps)


def _join_formula(s, to):
    z, x = s["branch"].to(to), s["resid"].to(to)
    a, _ = _act(s["gate"].to(to) if s["gate"] is not None else None, s["case"]["act"])
    out = x + s["scale"].to(to) * a * (z * _rms(z) * s["post_weight"].to(to))
    return {"out": out, "normed": out * _rms(out) * s["pre_weight"].to(to)}


def _join_plain(s):
    return {k: v.to(s["resid"].dtype) for k, v in _join_formula(s, torch.float32).items()}


def _join_grad_plain(s):
    f = torch.float32
    z, out, dy = s["branch"].to(f), s["out"].to(f), s["d_normed"].to(f)
    gate, act, w, c, u = s["gate"], s["case"]["act"], s["post_weight"], s["scale"], s["pre_weight"]
    a, da = _act(gate.to(f) if gate is not None else None, act)
    rz, ro = _rms(z), _rms(out)
    e = dy * u
    dx = s["d_out"].to(f) + ro * e - out * ro ** 3 * (e * out).mean(-1, keepdim=True)
    n = z * rz                                                # out = resid + c a w n
    k = dx * c * a * w
    t = s["branch"].dtype
    dxn = dx * n
    return {"d_branch": (rz * k - z * rz ** 3 * (k * z).mean(-1, keepdim=True)).to(t), "d_resid": dx.to(t),
            "d_gate": (dxn * c * w * da).to(t) if gate is not None else None,
            "d_post_weight": (dxn * c * a).sum(0), "d_scale": (dxn * a * w).sum(0), "d_pre_weight": (dy * out * ro).sum(0)}


def _step_plain(s):
    q = 1 / (1 + torch.exp(s["forget"].float() + s["bias"]))
    s["state"].copy_((1 - q) * s["state"] + q * s["value"].float())
    return {"hidden": s["state"].to(s["value"].dtype), "state": s["state"]}


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis, by doubling: after k rounds a row holds the last 2^k steps up to it."""
    n = 1
    while n < a.shape[0]:
        b = torch.cat([b[:n], b[n:] + a[n:] * b[:-n]])
        a = torch.cat([a[:n], a[n:] * a[:-n]])
        n *= 2
    return b


def _recurrence_plain(s):
    x, bias, n = s["value"].float(), s["bias"], s["value"].shape[0]
    q = 1 / (1 + torch.exp(s["forget"].float() + bias))
    a = 1 - q
    at = s["offsets"].long()
    full = (at[1:] > at[:-1]).nonzero()[:, 0]                 # sequences that have a step
    first, last = at[full], at[full + 1] - 1
    h0 = s["initial"]
    b = q * x
    b[first] += a[first] * h0[full]
    coef = a.clone()
    coef[first] = 0
    h = _scan(coef, b)
    final = h0.clone()
    final[full] = h[last]
    before = torch.cat([h0[:1], h[:-1]])
    before[first] = h0[full]
    # the same recurrence backwards: the gradient of h_t takes that of h_{t+1} times 1 - q_{t+1}
    d = s["d_hidden"].to(torch.float32, copy=True)
    d[last] += s["d_final"][full]
    back = torch.cat([a[1:], a[:1]])
    back[last] = 0
    d = _scan(back.flip(0), d.flip(0)).flip(0)
    dz = (before - x) * q * a * d
    d_initial = s["d_final"].clone()
    d_initial[full] = (a * d)[first]
    t = s["value"].dtype
    return {"hidden": h.to(t), "final": final, "d_value": (q * d).to(t), "d_forget": dz.to(t), "d_initial": d_initial, "d_bias": dz.sum(0)}


def _bits(n, update, seed, device):
    """Two random numbers of 16 bits for every place of a tensor."""
    mask = 0xFFFFFFFF
    key = (seed * 0xBB67AE85 + update * 0x9E3779B9) & mask
    x = (torch.arange(n, device=device) * 0x9E3779B9 + key) & mask
    x = (((x ^ (x >> 16)) & mask) * 0x6A09E667) & mask
    x = (((x ^ (x >> 15)) & mask) * 0x3C6EF373) & mask
    x = x ^ (x >> 16)
    return x & 0xFFFF, x >> 16


def _blocks(x):
    """A flat tensor as rows of BLOCK values, padded with zeros."""
    n = x.numel()
    return torch.cat([x.reshape(-1), x.new_zeros(-n % BLOCK)]).view(-1, BLOCK)


def _encode(x, chance):
    """Codes (as values) and scales of a flat tensor in 32 bits; `chance`: a number below 2^16 for every value."""
    rows = _blocks(x)
    top = rows.abs().amax(1, keepdim=True)
    top = torch.where(top < 1e-30, torch.zeros_like(top), top)
    y = (rows.abs() * torch.where(top > 0, LARGEST / top, torch.zeros_like(top))).clamp(max=LARGEST)
    r = _blocks(chance.int())
    normal = ((y.view(torch.int32) + (r << 4)) & ~0xFFFFF).view(torch.float32)      # 3 bits behind the leading one stay
    small = torch.floor(y * 512 + r * (1 / 65536)) * (1 / 512)                      # below 2^-6: multiples of 2^-9
    code = torch.where(y >= 1 / 64, normal, small).clamp(max=LARGEST)
    return torch.copysign(code, rows).view(-1)[: x.numel()], (top * (1 / LARGEST)).view(-1)


def _adamw_plain(s):
    case, t = s["case"], s["update"]
    c1, c2 = LR / (1 - BETA1 ** t), 1 / math.sqrt(1 - BETA2 ** t)
    for i, p in enumerate(s["p"]):
        g = s["g"][i].float().view(-1) * s["grad_scale"]
        flat, m, v = p.view(-1), s["m"][i].view(-1), s["v"][i].view(-1)
        n = flat.numel()
        if case["bits"] == 8:
            m = (_blocks(m.float()) * s["m_scale"][i][:, None]).view(-1)[:n]
            v = (_blocks(v.float()) * s["v_scale"][i][:, None]).view(-1)[:n].square()
        m = m * BETA1 + g * (1 - BETA1)
        v = v * BETA2 + (g * (1 - BETA2)) * g
        r = torch.sqrt(v)
        flat.copy_(flat * (1 - LR * DECAY) - m * c1 / (r * c2 + ADAM_EPS))
        if case["bits"] == 8:
            low, high = _bits(n, t, s["seed"], p.device)
            code, s["m_scale"][i][:] = _encode(m, low)
            s["m"][i].view(-1).copy_(code.to(torch.float8_e4m3fn))
            code, s["v_scale"][i][:] = _encode(r, high)
            code = torch.where((r > 0) & (s["v_scale"][i].repeat_interleave(BLOCK)[:n] > 0), code.clamp(min=1 / 512), code)
            s["v"][i].view(-1).copy_(code.to(torch.float8_e4m3fn))
        else:
            s["m"][i].view(-1).copy_(m)
            s["v"][i].view(-1).copy_(v)
        if s["copy"] is not None:
            s["copy"][i].copy_(p)
    return s["flat"]                                          # the tensors' own memory


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"join": _join_exact, "join_grad": _join_grad_exact, "step": _step_exact, "recurrence": _recurrence_exact, "adamw": _adamw_exact}[case["kind"]](s)


def _double(s, *names):
    return [s[k].double() if s[k] is not None else None for k in names]


def _join_exact(s):
    z, x, g, w, c, u = _double(s, "branch", "resid", "gate", "post_weight", "scale", "pre_weight")
    act = s["case"]["act"]
    a = {"none": lambda: torch.ones_like(z), "identity": lambda: g, "logistic": lambda: torch.sigmoid(g), "silu": lambda: g * torch.sigmoid(g)}[act]()
    out = x + c * a * w * z / torch.sqrt(z.square().mean(1, keepdim=True) + EPS)
    return {"out": out, "normed": u * out / torch.sqrt(out.square().mean(1, keepdim=True) + EPS)}


def _norm_grad(d, z):
    """Gradient of z / r, r = sqrt(mean(z^2) + eps), for the gradient d of the result; and z / r."""
    r = torch.sqrt(z.square().mean(1, keepdim=True) + EPS)
    n = z / r
    return (d - n * (d * n).mean(1, keepdim=True)) / r, n


def _join_grad_exact(s):
    z, out, g, w, c, u, d_out, dy = _double(s, "branch", "out", "gate", "post_weight", "scale", "pre_weight", "d_out", "d_normed")
    act = s["case"]["act"]
    d, n_out = _norm_grad(dy * u, out)
    d_pre, dx = (dy * n_out).sum(0), d_out + d
    a, da = torch.ones_like(z), None
    if act == "identity":
        a, da = g, torch.ones_like(z)
    elif act != "none":
        sig = torch.sigmoid(g)
        a, da = (sig, sig * torch.sigmoid(-g)) if act == "logistic" else (g * sig, sig + g * sig * torch.sigmoid(-g))
    d_branch, n = _norm_grad(dx * (c * w) * a, z)
    return {"d_branch": d_branch, "d_resid": dx, "d_gate": None if da is None else dx * (c * w) * n * da,
            "d_post_weight": c * (dx * n * a).sum(0), "d_scale": w * (dx * n * a).sum(0), "d_pre_weight": d_pre}


def _step_exact(s):
    x, f, b, h = _double(s, "value", "forget", "bias", "state")
    q = torch.sigmoid(-(f + b))
    h = h + q * (x - h)
    return {"hidden": h, "state": h}


def _recurrence_exact(s):
    """Step by step, one sequence after the other."""
    x, f, b, d_hidden, h0, d_final = _double(s, "value", "forget", "bias", "d_hidden", "initial", "d_final")
    q, a = torch.sigmoid(-(f + b)), torch.sigmoid(f + b)
    h, before, d, b_t = torch.empty_like(x), torch.empty_like(x), d_hidden, q * x
    final, d_initial = h0.clone(), d_final.clone()
    at = s["offsets"].tolist()
    a_row, b_row, h_row, d_row = a.unbind(0), b_t.unbind(0), h.unbind(0), d.unbind(0)
    for i, (begin, end) in enumerate(zip(at, at[1:])):
        if begin == end:
            continue
        state = h0[i]
        for t in range(begin, end):
            state = torch.addcmul(b_row[t], a_row[t], state, out=h_row[t])
        final[i] = state
        before[begin], before[begin + 1:end] = h0[i], h[begin:end - 1]
        d_row[end - 1].add_(d_final[i])
        for t in range(end - 1, begin, -1):
            d_row[t - 1].addcmul_(a_row[t], d_row[t])
        d_initial[i] = a_row[begin] * d_row[begin]
    d_forget = d * q * a * (before - x)
    return {"hidden": h, "final": final, "d_value": d * q, "d_forget": d_forget, "d_initial": d_initial, "d_bias": d_forget.sum(0)}


def _adamw_exact(s):
    case, t, out = s["case"], s["update"], {k: v.double() for k, v in s["flat"].items()}
    place = 0
    for g in s["g"]:
        n = g.numel()
        here, place = slice(place, place + n), place + -(-n // BLOCK) * BLOCK
        blocks = slice(here.start // BLOCK, place // BLOCK)
        each = torch.arange(n, device=g.device) // BLOCK
        g = g.double().reshape(-1) * s["grad_scale"].double()
        m, root = out["m"][here], out["v"][here]
        if case["bits"] == 8:
            m, root = m * out["m_scale"][blocks][each], root * out["v_scale"][blocks][each]
        v = root ** 2 if case["bits"] == 8 else root
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
        p = out["p"][here]
        p -= LR * (DECAY * p + m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS))
        if "copy" in out:
            out["copy"][here] = p
        if case["bits"] == 32:
            out["m"][here], out["v"][here] = m, v
            continue
        x = (torch.arange(n, device=g.device) * 0x9E3779B9 + s["seed"] * 0xBB67AE85 + t * 0x9E3779B9) % 2 ** 32
        x = (x ^ x // 2 ** 16) * 0x6A09E667 % 2 ** 32
        x = (x ^ x // 2 ** 15) * 0x3C6EF373 % 2 ** 32
        x = x ^ x // 2 ** 16
        for name, y, chance in (("m", m, x % 2 ** 16), ("v", v.sqrt(), x // 2 ** 16)):
            top = torch.zeros(blocks.stop - blocks.start, dtype=y.dtype, device=y.device).scatter_reduce(0, each, y.abs(), "amax")
            scale = top / LARGEST
            ratio = y.abs() / scale[each]
            step = 2.0 ** (torch.frexp(ratio)[1].clamp(min=-5) - 4)      # distance of the codes about a value in [2^e, 2^(e+1)): 2^(e-3)
            code = step * torch.floor(ratio / step + chance / 65536)
            code = torch.where(ratio >= LARGEST * (1 - 1e-12), torch.full_like(code, LARGEST), code)
            if name == "v":
                code = torch.where(y > 0, code.clamp(min=2.0 ** -9), code)
            out[name][here], out[name + "_scale"][blocks] = torch.copysign(code, y), scale
    return out
