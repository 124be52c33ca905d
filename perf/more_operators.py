"""More operators of a policy with memory, as they are measured: what they compute in plain form, and the calls that compute it.

Blocks whose memory is a matrix for every head instead of a number for every channel, the norms they need, and the clipping of their
gradients.  A case is one call (or one forward and backward pass) of one operator, by `kind`:

  norm         layer norm of every row, or of each of `groups` equal parts of a row (the heads) on its own:
                 y = (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) * weight + bias
  norm_grad    its gradient with respect to x, weight and bias
  attend       linear attention with a decay for every head, over sequences of different lengths packed one after the other:
                 S_t = decay S_{t-1} + k_t v_t^T,   o_t = scale q_t S_t
               `heads` heads of queries share `states` heads of keys, values and memories S in equal parts
  attend_train the same, and its gradient with respect to queries, keys, values and the first S
  attend_step  one step of it for many sequences at once, S updated in place
  clip         the norm of the gradients of many tensors together, and the factor that brings it down to `max_norm`; with `write`, also the
               gradients times that factor
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
CLIP_EPS, MAX_NORM = 1e-6, 1.0
KINDS = ("norm", "norm_grad", "attend", "attend_train", "attend_step", "clip")


def listed():
    return [
        # a controller serving a few machines: one row each, so latency is all there is
        {"name": "norm_serve", "kind": "norm", "rows": 16, "width": 512, "groups": 1, "dtype": "bf16"},
        # the memories' answers of a training batch, every head on its own: 64 trajectories of 1000 steps
        {"name": "norm_heads", "kind": "norm", "rows": 64000, "width": 1024, "groups": 16, "dtype": "f16"},
        # the backward pass of a large batch through a wide block
        {"name": "norm_grad_large", "kind": "norm_grad", "rows": 65536, "width": 4096, "groups": 1, "dtype": "bf16"},
        # a width that fits no vector and no tile, in 32 bits
        {"name": "norm_grad_odd", "kind": "norm_grad", "rows": 9973, "width": 777, "groups": 1, "dtype": "f32"},
        # one control period of 256 machines
        {"name": "step_serve", "kind": "attend_step", "sequences": 256, "heads": 8, "states": 8, "key": 64, "value": 64, "dtype": "bf16"},
        # one machine, one control period
        {"name": "step_single", "kind": "attend_step", "sequences": 1, "heads": 8, "states": 8, "key": 64, "value": 64, "dtype": "bf16"},
        # a training batch: 64 trajectories of 1000 steps
        {"name": "attend_batch", "kind": "attend_train", "tokens": 64000, "sequences": 64, "lengths": "equal", "heads": 8, "states": 8,
         "key": 64, "value": 64, "dtype": "bf16"},
        # one very long recording read at once before a controller takes over; queries share memories; the only work to share out lies along it
        {"name": "attend_long", "kind": "attend", "tokens": 131072, "sequences": 1, "lengths": "equal", "heads": 8, "states": 2, "key": 128,
         "value": 128, "dtype": "bf16"},
        # episodes that ended at different times, some at once, packed one after the other; odd widths, in 32 bits
        {"name": "attend_packed", "kind": "attend_train", "tokens": 10007, "sequences": 61, "lengths": "ragged", "heads": 6, "states": 3,
         "key": 40, "value": 77, "dtype": "f32"},
        # the largest memoryless policy: six tensors of 1 to 65536 values
        {"name": "clip_policy", "kind": "clip", "sizes": "256x5,256,256x256,256,256,1", "repeat": 1, "grad": "f32", "write": False},
        # a policy of eight blocks, 64 tensors; the factor goes to the update, the gradients stay
        {"name": "clip_blocks", "kind": "clip", "sizes": "1024x1024,1024x1024,1024x1024,1024x1024,1024,1024,1024,1024", "repeat": 8, "grad": "bf16",
         "write": False},
        # a large model whose clipped gradients are kept; tensors of odd counts among them
        {"name": "clip_large", "kind": "clip", "sizes": "4096x4096,4096x4096,4096x4096,4093x4095,4096,777,1,4096", "repeat": 6, "grad": "bf16",
         "write": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return rng.choice([64, 64, 128, 128, _log_int(rng, 8, 128), _log_int(rng, 8, 128)])


def draw(rng):
    kind = rng.choice(KINDS)
    dtype = rng.choice(sorted(DTYPES))
    each = 2 if dtype == "f32" else 1
    if kind in ("norm", "norm_grad"):
        groups = rng.choice([1, 1, 1, 2, 8, _log_int(rng, 2, 32)])
        part = _log_int(rng, max(16, 64 // groups), 8192 // groups)
        if rng.random() < 0.5:
            part = min(8192 // groups, 2 ** round(math.log2(part)))
        width = groups * part
        rows = _log_int(rng, 1, 65536 * 4096 // (width * each))
        return {"kind": kind, "rows": min(rows, 262144), "width": width, "groups": groups, "dtype": dtype}
    if kind == "clip":
        repeat = _log_int(rng, 1, 24)
        total = _log_int(rng, 2000, 4e8 / each) // repeat
        sizes, count = [], rng.randint(1, 8)
        for _ in range(count):
            n = _log_int(rng, 1, max(1, total // count))
            if n > 4096 and rng.random() < 0.5:
                side = _log_int(rng, 16, n // 16)
                sizes.append("%dx%d" % (side, n // side))
            else:
                sizes.append(str(n))
        return {"kind": kind, "sizes": ",".join(sizes), "repeat": repeat, "grad": dtype, "write": rng.random() < 0.5}
    states = rng.choice([1, 2, 3, 4, 8, 8, 12])
    heads = states * rng.choice([1, 1, 1, 2, 4])
    key, value = _width(rng), _width(rng)
    if rng.random() < 0.5:
        value = key
    case = {"kind": kind, "heads": heads, "states": states, "key": key, "value": value, "dtype": dtype}
    if kind == "attend_step":
        case["sequences"] = _log_int(rng, 1, max(2, min(4096, 2 ** 27 // (states * key * value))))
        return case
    # no more entries than a third of the long recording's, as a pass in 32 bits or backwards takes a few times longer; and no row is narrower than 64
    most = 131072 * 8 * 256 // (3 * each * max(64, heads * (key + value)))
    tokens = _log_int(rng, 64, min(131072, most))
    sequences = _log_int(rng, 1, max(1, min(512, tokens // 16)))
    lengths = rng.choice(["equal", "ragged"])
    if lengths == "equal":
        tokens = max(1, tokens // sequences) * sequences
    case.update(tokens=tokens, sequences=sequences, lengths=lengths)
    return case


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
    if kind in ("norm", "norm_grad"):
        r, d, t = case["rows"], case["width"], DTYPES[case["dtype"]]
        s["x"] = normal(r, d, scale=2.0, mean=0.5, dtype=t)
        s["weight"], s["bias"] = normal(d, scale=0.1, mean=1.0), normal(d, scale=0.1)
        if kind == "norm_grad":
            s["d_out"] = normal(r, d, scale=1e-2, dtype=t)
        return s
    if kind == "clip":
        shapes = _shapes(case)
        t = DTYPES[case["grad"]]
        s["g"] = [normal(*sh, scale=1e-2, dtype=t) for sh in shapes]
        s["grad_scale"] = torch.full((1,), 0.37, device="cuda")
        if case["write"]:                                     # kept in one allocation, as a trainer holds them
            flat, at, s["out"] = torch.zeros(sum(math.prod(sh) for sh in shapes), dtype=t, device="cuda"), 0, []
            for sh in shapes:
                s["out"].append(flat[at:at + math.prod(sh)].view(sh))
                at += math.prod(sh)
            s["flat"] = flat
        return s
    h, n, dk, dv, t = case["heads"], case["states"], case["key"], case["value"], DTYPES[case["dtype"]]
    tokens, sequences = case["sequences"] if kind == "attend_step" else case["tokens"], case["sequences"]
    # queries, keys and values are parts of one projection, as a block makes them
    proj = normal(tokens, h * dk + n * (dk + dv), dtype=t)
    s["q"], s["k"] = proj[:, :h * dk].view(tokens, h, dk), proj[:, h * dk:(h + n) * dk].view(tokens, n, dk)
    s["v"] = proj[:, (h + n) * dk:].view(tokens, n, dv)
    s["scale"] = dk ** -0.5
    # memories of a few steps up to a few hundred
    s["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(2.0, 8.0, n, device="cuda")))
    if kind == "attend_step":
        s["state"] = normal(sequences, n, dk, dv, scale=2.0)
        return s
    s["initial"] = normal(sequences, n, dk, dv, scale=0.5)
    if kind == "attend_train":
        s["d_out"] = normal(tokens, h, dv, scale=1e-2, dtype=t)
        s["d_final"] = normal(sequences, n, dk, dv, scale=1e-2)
    s["offsets"] = torch.tensor(_offsets(case, torch.Generator().manual_seed(seed)), dtype=torch.int32, device="cuda")
    return s


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n, e, d = case["rows"] * case["width"], size[case["dtype"]], case["width"]
        return {"bytes": n * e * 2 + 8 * d, "flops": 9 * n} if kind == "norm" else {"bytes": n * e * 3 + 12 * d, "flops": 18 * n}
    if kind == "clip":
        n, e = sum(math.prod(sh) for sh in _shapes(case)), size[case["grad"]]
        return {"bytes": n * e * (2 if case["write"] else 1) + 12, "flops": n * (3 if case["write"] else 2)}
    h, n, dk, dv, e = case["heads"], case["states"], case["key"], case["value"], size[case["dtype"]]
    moved, state = (h + n) * (dk + dv) * e, n * dk * dv
    if kind == "attend_step":
        return {"bytes": case["sequences"] * (moved + 8 * state) + 4 * n, "flops": case["sequences"] * (3 * state + 2 * h * dk * dv)}
    # the recurrence itself: products of a row with the memory, and the memory's update
    t, read = case["tokens"], 8 * state * case["sequences"] + 4 * n
    if kind == "attend":
        return {"bytes": t * moved + read, "flops": t * (3 * state + 2 * h * dk * dv)}
    # forward (q, k, v read, o written) and back (q, k, v, do read, dq, dk, dv written), with what both read counted once
    return {"bytes": t * 2 * moved + 2 * read, "flops": 3 * t * (3 * state + 2 * h * dk * dv)}


# ------------------------------------------------------------------------------------------------ the calls, and the plain forms
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"norm": _norm_own, "norm_grad": _norm_grad_own, "attend": _attend_own, "attend_train": _attend_own, "attend_step": _step_own,
                "clip": _clip_own}[kind](s)
    return {"norm": _norm_plain, "norm_grad": _norm_grad_plain, "attend": _attend_plain, "attend_train": _attend_plain, "attend_step": _step_plain,
            "clip": _clip_plain}[kind](s)


def _norm_own(s):
    from paper_2202_13638_amd import binding
    out = torch.empty_like(s["x"])
    binding.bagel_layer_norm(s["x"], out, weight=s["weight"], bias=s["bias"], groups=s["case"]["groups"], eps=EPS)
    return {"out": out}


def _norm_grad_own(s):
    from paper_2202_13638_amd import binding
    r = {"d_x": torch.empty_like(s["x"]), "d_weight": torch.empty_like(s["weight"]), "d_bias": torch.empty_like(s["bias"])}
    binding.bagel_layer_norm_grad(s["x"], s["d_out"], weight=s["weight"], groups=s["case"]["groups"], eps=EPS, **r)
    return r


def _attend_own(s):
    from paper_2202_13638_amd import binding
    t, h, n, dk, dv = (*s["q"].shape[:2], *s["initial"].shape[1:])
    new, dtype = s["q"].new_empty, s["q"].dtype
    r = {"out": new(t, h, dv), "final": torch.empty_like(s["initial"])}
    binding.bagel_linear_attention(s["q"], s["k"], s["v"], r["out"], s["offsets"], s["log_decay"], scale=s["scale"], initial=s["initial"],
                                   final=r["final"])
    if s["case"]["kind"] == "attend_train":
        r.update(d_query=new(t, h, dk, dtype=dtype), d_key=new(t, n, dk, dtype=dtype), d_value=new(t, n, dv, dtype=dtype),
                 d_initial=torch.empty_like(s["initial"]))
        binding.bagel_linear_attention_grad(s["q"], s["k"], s["v"], s["d_out"], r["d_query"], r["d_key"], r["d_value"], s["offsets"], s["log_decay"],
                                            scale=s["scale"], initial=s["initial"], d_final=s["d_final"], d_initial=r["d_initial"])
    return r


def _step_own(s):
    from paper_2202_13638_amd import binding
    out = s["q"].new_empty(*s["q"].shape[:2], s["case"]["value"])
    binding.bagel_linear_attention_step(s["q"], s["k"], s["v"], s["state"], out, s["log_decay"], scale=s["scale"])
    return {"out": out, "state": s["state"]}


def _clip_own(s):
    from paper_2202_13638_amd import binding
    r = {"norm": torch.empty(1, device="cuda"), "factor": torch.empty(1, device="cuda")}
    binding.bagel_clip_norm(s["g"], MAX_NORM, r["norm"], r["factor"], grad_scale=s["grad_scale"], out=s.get("out"), eps=CLIP_EPS)
    if "out" in s:
        r["flat"] = s["flat"]                                 # the written gradients' own memory
    return r


def _parts(s, x):
    return x.float().view(x.shape[0], s["case"]["groups"], -1)


def _centred(x):
    """x less its mean, and one over its standard deviation."""
    c = x - x.mean(-1, keepdim=True)
    return c, torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)


def _norm_plain(s):
    c, r = _centred(_parts(s, s["x"]))
    return {"out": ((c * r).view(s["x"].shape) * s["weight"] + s["bias"]).to(s["x"].dtype)}


def _norm_grad_plain(s):
    c, r = _centred(_parts(s, s["x"]))
    n, d = c * r, s["d_out"].float()
    e = (d * s["weight"]).view(n.shape)
    dx = r * (e - e.mean(-1, keepdim=True) - n * (e * n).mean(-1, keepdim=True))
    return {"d_x": dx.view(s["x"].shape).to(s["x"].dtype), "d_weight": (d * n.view(d.shape)).sum(0), "d_bias": d.sum(0)}


CHUNK = 64


class _Packed:
    """Packed rows as chunks of CHUNK of every sequence: forwards, or backwards from each sequence's end."""

    def __init__(self, s, back):
        at = s["offsets"].long()
        length = at[1:] - at[:-1]
        case = s["case"]
        most = case["tokens"] // case["sequences"] if case["lengths"] == "equal" else int(length.max())
        self.chunks = max(1, -(-most // CHUNK))
        m = torch.arange(self.chunks * CHUNK, device=at.device)
        self.here = m < length[:, None]                       # [sequence, place]
        self.rows = torch.where(self.here, at[1:, None] - 1 - m if back else at[:-1, None] + m, 0)
        self.count = (length[:, None] - m[::CHUNK]).clamp(0, CHUNK).float()      # rows of every chunk

    def take(self, x, states):
        """[rows, heads, width] -> [sequence, chunk, memory, heads of it * place, width]; zeros where there is no row."""
        x = x.float()[self.rows] * self.here[..., None, None]
        n, _, h, d = x.shape
        x = x.view(n, self.chunks, CHUNK, states, h // states, d)
        return x.permute(0, 1, 3, 4, 2, 5).reshape(n, self.chunks, states, h // states * CHUNK, d)

    def put(self, x, like):
        n, c, states, gm, d = x.shape
        x = x.view(n, c, states, gm // CHUNK, CHUNK, d).permute(0, 1, 4, 2, 3, 5).reshape(n, c * CHUNK, -1, d)
        out = torch.zeros(like.shape[0], *x.shape[2:], device=like.device)
        out[self.rows[self.here]] = x[self.here]
        return out.to(like.dtype)


def _attend_chunks(p, q, k, v, log_decay, first, back):
    """o of q, k, v in chunks, and the memory behind the last: `first` [sequence, memory, key, value] is the one before.

    Where several heads of queries share a memory, k and v may have the one head, or (in the backward pass) as many as q had."""
    device = q.device
    m = torch.arange(CHUNK, device=device)
    ln = log_decay[:, None]                                   # [memory, place]
    behind = (p.count[:, :, None, None] - 1 - m + (1 if back else 0)).clamp(min=0)       # rows from one to the end of its chunk
    # what a chunk adds to the memory, and the memory before each
    rows_k = k.shape[3] // CHUNK
    weight = torch.exp(ln * behind).repeat(1, 1, 1, rows_k)
    add = torch.matmul((k * weight[..., None]).transpose(-1, -2), v)
    keep = torch.exp(log_decay[None, None] * p.count[:, :, None])[..., None, None]
    memory, before = first, torch.empty_like(add)
    for c in range(p.chunks):
        before[:, c] = memory
        memory = keep[:, c] * memory + add[:, c]
    # rows of one chunk with each other
    gap = m[:, None] - m[None, :]
    mask = torch.where(gap >= 0, torch.exp(log_decay[:, None, None] * gap.clamp(min=0)), torch.zeros((), device=device))
    mask = mask.repeat(1, q.shape[3] // CHUNK, rows_k)
    inter = torch.exp(ln * (m + (0 if back else 1))).repeat(1, q.shape[3] // CHUNK)
    o = torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * mask, v) + torch.matmul(q * inter[..., None], before)
    return o, memory


def _attend_plain(s):
    n, ld = s["case"]["states"], s["log_decay"]
    p = _Packed(s, False)
    q, k, v = p.take(s["q"], n) * s["scale"], p.take(s["k"], n), p.take(s["v"], n)
    o, final = _attend_chunks(p, q, k, v, ld, s["initial"], False)
    r = {"out": p.put(o, s["q"]), "final": final}
    if s["case"]["kind"] == "attend":
        return r
    # the gradient of the queries reads a memory of values and keys; those of keys and values one that runs backwards
    do = p.take(s["d_out"], n)
    r["d_query"] = p.put(_attend_chunks(p, do, v, k, ld, s["initial"].transpose(-1, -2), False)[0] * s["scale"], s["q"])
    p = _Packed(s, True)
    q, k, v, do = p.take(s["q"], n) * s["scale"], p.take(s["k"], n), p.take(s["v"], n), p.take(s["d_out"], n)
    r["d_key"] = p.put(_attend_chunks(p, v, do, q, ld, s["d_final"].transpose(-1, -2), True)[0], s["q"])
    dv, r["d_initial"] = _attend_chunks(p, k, q, do, ld, s["d_final"], True)
    r["d_value"] = p.put(dv, s["q"])
    return r


def _step_plain(s):
    n, (t, h, dk) = s["case"]["states"], s["q"].shape
    s["state"].mul_(torch.exp(s["log_decay"])[:, None, None]).add_(s["k"].float()[..., None] * s["v"].float()[..., None, :])
    q = s["q"].float().view(t, n, h // n, dk) * s["scale"]
    return {"out": torch.matmul(q, s["state"]).view(t, h, -1).to(s["q"].dtype), "state": s["state"]}


def _clip_plain(s):
    sums = [g.float().square().sum(dtype=torch.float64) for g in s["g"]]
    norm = (torch.stack(sums).sum().sqrt() * s["grad_scale"].abs()).float()
    factor = s["grad_scale"] * (MAX_NORM / (norm + CLIP_EPS)).clamp(max=1.0)
    r = {"norm": norm, "factor": factor}
    if "out" in s:
        for g, out in zip(s["g"], s["out"]):
            out.copy_(g.float() * factor)
        r["flat"] = s["flat"]                                 # the written gradients' own memory
    return r


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "norm_grad": _norm_exact, "attend": _attend_exact, "attend_train": _attend_exact, "attend_step": _step_exact,
            "clip": _clip_exact}[case["kind"]](s)


def _norm_exact(s):
    grad = s["case"]["kind"] == "norm_grad"
    size, width = s["case"]["width"] // s["case"]["groups"], s["case"]["width"]
    weight, bias = s["weight"].double(), s["bias"].double()
    out, dw, db = [], torch.zeros_like(weight), torch.zeros_like(weight)
    for i in range(0, s["x"].shape[0], 16384):                # some rows at a time
        x = s["x"][i:i + 16384].double().reshape(-1, size)
        x = (x - x.sum(1, keepdim=True) / size)
        dev = (x.pow(2).sum(1, keepdim=True) / size + EPS).sqrt()
        y = (x / dev).view(-1, width)
        if not grad:
            out.append(y * weight + bias)
            continue
        d = s["d_out"][i:i + 16384].double()
        dw += (d * y).sum(0)
        db += d.sum(0)
        e, y = (d * weight).view(-1, size), y.view(-1, size)
        out.append(((e - e.sum(1, keepdim=True) / size - y * ((e * y).sum(1, keepdim=True) / size)) / dev).view(-1, width))
    out = torch.cat(out)
    return {"d_x": out, "d_weight": dw, "d_bias": db} if grad else {"out": out}


def _attend_exact(s):
    """Every sequence on its own, as the sum over all pairs of rows, some hundred rows at a time; gradients by torch from that."""
    case, train = s["case"], s["case"]["kind"] == "attend_train"
    group, at, ln = case["heads"] // case["states"], s["offsets"].tolist(), s["log_decay"].double()
    longest = max(b - a for a, b in zip(at, at[1:]))
    if longest > 200000 or case["sequences"] > 2000:
        return None
    part = 512
    gap = torch.arange(part, device="cuda", dtype=torch.float64)
    gap = gap[:, None] - gap
    pairs = torch.where(gap < 0, 0.0, torch.pow(torch.exp(ln)[:, None, None], gap.clamp(min=0)))
    out = {"out": s["q"].new_zeros(*s["q"].shape[:2], case["value"], dtype=torch.float64), "final": s["initial"].double()}
    if train:
        out.update(d_query=torch.zeros_like(s["q"], dtype=torch.float64).contiguous(), d_key=torch.zeros_like(s["k"], dtype=torch.float64).contiguous(),
                   d_value=torch.zeros_like(s["v"], dtype=torch.float64).contiguous(), d_initial=s["d_final"].double())
    for i, (begin, end) in enumerate(zip(at, at[1:])):
        if begin == end:
            continue
        with torch.set_grad_enabled(train):
            leaves = [s[k][begin:end].double().transpose(0, 1).contiguous().requires_grad_(train) for k in ("q", "k", "v")]
            memory = first = s["initial"][i].double().requires_grad_(train)
            q, k, v = leaves[0] * s["scale"], leaves[1].repeat_interleave(group, 0), leaves[2].repeat_interleave(group, 0)
            o = []
            for a in range(0, end - begin, part):
                n = min(part, end - begin - a)
                qa, ka, va = q[:, a:a + n], k[:, a:a + n], v[:, a:a + n]
                steps = torch.arange(1, n + 1, device="cuda", dtype=torch.float64)
                decay = torch.exp(ln)[:, None].pow(steps)                                  # [memory, row]
                seen = (qa @ ka.transpose(1, 2).contiguous()) * pairs[:, :n, :n].repeat_interleave(group, 0)
                o.append(seen @ va + decay.repeat_interleave(group, 0)[..., None] * (qa @ memory.repeat_interleave(group, 0)))
                left = torch.exp(ln)[:, None].pow(n - steps)[..., None]
                own_k, own_v = leaves[1][:, a:a + n], leaves[2][:, a:a + n]
                memory = decay[:, -1, None, None] * memory + (own_k * left).transpose(1, 2).contiguous() @ own_v
            o = torch.cat(o, 1)
            if train:
                d = torch.autograd.grad([o, memory], [*leaves, first], [s["d_out"][begin:end].double().transpose(0, 1), s["d_final"][i].double()])
                for key, x in zip(("d_query", "d_key", "d_value"), d):
                    out[key][begin:end] = x.transpose(0, 1)
                out["d_initial"][i] = d[3]
            out["out"][begin:end] = o.detach().transpose(0, 1)
            out["final"][i] = memory.detach()
    return out


def _step_exact(s):
    group, decay = s["case"]["heads"] // s["case"]["states"], torch.exp(s["log_decay"].double())
    k, v = s["k"].double(), s["v"].double()
    state = decay.view(-1, 1, 1) * s["state"].double() + k.unsqueeze(-1) * v.unsqueeze(-2)
    q = s["q"].double() * s["scale"]
    out = torch.stack([(q[:, h, :, None] * state[:, h // group]).sum(1) for h in range(q.shape[1])], 1)
    return {"out": out, "state": state}


def _clip_exact(s):
    scale = s["grad_scale"].double()
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["g"]:
        for part in g.reshape(-1).split(1 << 26):
            part = part.double() * scale
            total += torch.dot(part, part)
    norm = total.sqrt()
    factor = scale * torch.minimum(torch.ones_like(norm), MAX_NORM / (norm + CLIP_EPS))
    r = {"norm": norm, "factor": factor}
    if "out" in s:
        r["flat"] = torch.cat([g.reshape(-1) for g in s["g"]]).double() * factor
    return r
