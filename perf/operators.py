"""Operators of a Peri-LN decoder's training step, and the calls that they are judged by.

  adamw    one AdamW step of M replicas of a tensor list, states in 8 bits or in
           32 (``clip``: after the clip of each replica's gradient to norm 1)
  average  the mean over the replicas of parameters, m and v, as a period's end asks
  fwd      the residual update between two blocks: the norm after a block, its gate,
           the scaled residual, the norm before the next block
  bwd      the gradients of that update

Tensor lists: the decoder lists of the synthetic workloads, a small MLP, uneven
pieces of odd totals.  Rows: sequences of 2048 tokens at the lists' widths, a few
tokens, odd counts.  ``listed`` names what each case stands for.
"""
import math
import random

import torch

own = False

BETAS = (0.9, 0.999)
EPS = 1e-8
DECAY = 0.1
LR = 1e-4
RHO = 1.0
SEED = 20251007
T0 = 1024                 # steps already taken
BLOCK = 256               # elements that share a scale
SIGMA = 1e-3              # gradient scale of the decoder workloads
NORM_EPS = 1e-5
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    small_gpt = {"vocab": 50257, "d": 768, "ffn": 3072, "blocks": 12}
    large = {"vocab": 50257, "d": 2048, "ffn": 8192, "blocks": 24}
    return [
        # the MLP of a unit test, four workers: latency of the call
        {"name": "adamw-mlp-m4-8bit", "op": "adamw", "M": 4, "bits": 8, "param": "f32", "grad": "f32",
         "numel": 2632, "tensors": 4, "clip": False, "shift": 0},
        # a GPT-2-small-shaped list trained by four workers in bf16, clipped at 1
        {"name": "adamw-gpt2-m4-8bit-clip", "op": "adamw", "M": 4, "bits": 8, "param": "bf16", "grad": "bf16",
         "clip": True, "shift": 0, **small_gpt},
        # fp32 parameters and states with bf16 gradients, two workers
        {"name": "adamw-gpt2-m2-32bit", "op": "adamw", "M": 2, "bits": 32, "param": "f32", "grad": "bf16",
         "clip": False, "shift": 0, **small_gpt},
        # one worker's ~1B list
        {"name": "adamw-1b-8bit", "op": "adamw", "M": 1, "bits": 8, "param": "bf16", "grad": "bf16",
         "clip": False, "shift": 0, **large},
        # uneven pieces that start at odd addresses, clipped
        {"name": "adamw-5m-m3-odd", "op": "adamw", "M": 3, "bits": 8, "param": "f32", "grad": "bf16",
         "numel": 5000011, "tensors": 9, "clip": True, "shift": 1},
        # the end of a period: four replicas of the GPT-2-small list, all states
        {"name": "average-gpt2-m4-8bit", "op": "average", "M": 4, "bits": 8, "param": "bf16", "shift": 0, **small_gpt},
        # eight workers of a ragged list in 32 bits
        {"name": "average-5m-m8-32bit", "op": "average", "M": 8, "bits": 32, "param": "f32",
         "numel": 5000011, "tensors": 9, "shift": 0},
        # a few tokens of a GPT-2-small-sized model (generation): latency
        {"name": "fwd-4x768", "op": "fwd", "rows": 4, "d": 768, "norm": "layer", "bias": True, "gate": "none",
         "stream": "bf16", "branch": "bf16", "extra": 0},
        # four sequences of 2048 in mixed precision, per-channel gate
        {"name": "fwd-8192x768-mixed", "op": "fwd", "rows": 8192, "d": 768, "norm": "layer", "bias": True,
         "gate": "channel", "stream": "f32", "branch": "bf16", "extra": 0},
        # 32 sequences of 2048 at the ~1B list's width
        {"name": "fwd-65536x2048", "op": "fwd", "rows": 65536, "d": 2048, "norm": "rms", "bias": False,
         "gate": "channel", "stream": "bf16", "branch": "bf16", "extra": 0},
        # odd rows and an odd width, one gate row a sequence of 53 (conditioning per sequence)
        {"name": "bwd-1537x1001-odd", "op": "bwd", "rows": 1537, "d": 1001, "norm": "layer", "bias": True,
         "gate": "sequence", "groups": 29, "stream": "f32", "branch": "f32", "extra": 3},
        # 16 sequences of 2048 at the ~1B list's width
        {"name": "bwd-32768x2048", "op": "bwd", "rows": 32768, "d": 2048, "norm": "rms", "bias": False,
         "gate": "channel", "stream": "bf16", "branch": "bf16", "extra": 0},
    ]


def draw(rng):
    op = rng.choice(["adamw", "adamw", "average", "fwd", "fwd", "bwd", "bwd"])
    if op in ("adamw", "average"):
        M = rng.choice([1, 2, 3, 4, 6, 8, 12, 16] if op == "adamw" else [2, 3, 4, 5, 8, 12, 16, 32])
        numel = max(8, int(2 ** rng.uniform(7.0, 28.5) / M))
        if rng.random() < 0.5:
            numel |= 1
        case = {"op": op, "M": M, "bits": rng.choice([8, 8, 32]), "param": rng.choice(["f32", "bf16"]),
                "numel": numel, "tensors": min(1 + numel // 8, int(2 ** rng.uniform(0.0, 8.0))),
                "shift": rng.choice([0, 0, 0, 1, 8])}
        if op == "adamw":
            case |= {"grad": rng.choice(["f32", "bf16"]), "clip": rng.random() < 0.4}
        return case
    rows = int(2 ** rng.uniform(0.0, 16.0))
    d = rng.choice([64, 128, 256, 384, 512, 768, 1024, 1536, 2048, 4096, 8192, int(2 ** rng.uniform(3.0, 13.0))])
    rows = max(1, min(rows, 10 ** 8 // d))
    gate = rng.choice(["none", "channel", "channel", "sequence", "element"])
    stream, branch = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16")])
    norm = rng.choice(["rms", "layer"])
    case = {"op": op, "rows": rows, "d": d, "norm": norm, "bias": norm == "layer" and rng.random() < 0.7, "gate": gate,
            "stream": stream, "branch": branch, "extra": rng.choice([0, 0, 0, 8, 64, 3])}
    if gate == "sequence":
        case["groups"] = rng.choice([k for k in range(1, min(rows, 64) + 1) if rows % k == 0])
    return case


# ------------------------------------------------------------------ inputs

def _numels(case):
    """The case's tensor list: a decoder's (embedding, then per block qkv, proj,
    fc1, fc2 and four norm vectors, then the final norm), or ``numel`` elements
    cut into ``tensors`` uneven pieces."""
    if "blocks" in case:
        d, ffn = case["d"], case["ffn"]
        block = [3 * d * d, d * d, d * ffn, ffn * d, d, d, d, d]
        return [case["vocab"] * d] + block * case["blocks"] + [d, d]
    rng = random.Random(case["numel"])
    cuts = sorted(rng.sample(range(1, case["numel"]), case["tensors"] - 1)) if case["tensors"] > 1 else []
    edges = [0] + cuts + [case["numel"]]
    return [b - a for a, b in zip(edges, edges[1:])]


def _places(case):
    """(offset, numel, decay factor) of each tensor in a replica's vector, whose
    tensors start at multiples of BLOCK, and that vector's length.  Matrices
    decay, vectors and small tensors do not."""
    places, at = [], 0
    for k in _numels(case):
        places.append((at, k, 1.0 if k > 8192 else 0.0))
        at += -(-k // BLOCK) * BLOCK
    return places, at


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _vector(case, dtype, n):
    """[M][n] zeros that start ``shift`` elements after an aligned address."""
    M, shift = case["M"], case["shift"]
    return torch.zeros((M * n + shift,), device="cuda", dtype=dtype)[shift:].view(M, n)


def _zero_padding(t, places):
    """Clears what lies between the tensors of a replica's vector."""
    for (at, k, _), end in zip(places, [p[0] for p in places[1:]] + [t.shape[-1]]):
        if at + k < end:
            t[..., at + k:end].zero_()


def _adamw_inputs(case, gen, places, n):
    """Parameters, gradients, m and v of a run under way, [M][n]: replicas apart by
    a little, gradients with one position in a hundred 100 times larger, v of the
    gradients' scale."""
    p = _vector(case, KINDS[case["param"]], n)
    base = torch.empty((n,), device="cuda").normal_(0.0, 0.02, generator=gen)
    for row in p:
        row.copy_(torch.empty_like(base).normal_(0.0, 1e-3, generator=gen).add_(base))
    far = torch.where(torch.rand((n,), device="cuda", generator=gen) < 0.01, 100.0, 1.0)
    g = None
    if case["op"] == "adamw":
        g = _vector(case, KINDS[case["grad"]], n)
        for row in g:
            row.copy_(torch.empty_like(far).normal_(0.0, SIGMA, generator=gen).mul_(far))
    m = torch.empty((case["M"], n), device="cuda").normal_(0.0, 0.2 * SIGMA, generator=gen).mul_(far)
    v = torch.empty((case["M"], n), device="cuda").uniform_(0.25 * SIGMA ** 2, 2.0 * SIGMA ** 2, generator=gen)
    v.mul_(far).mul_(far)
    for t in (p, m, v) if g is None else (p, g, m, v):
        _zero_padding(t, places)
    return p, g, m, v


def _rows_tensor(case, dtype, gen, scale=1.0):
    """[rows][d], the rows ``extra`` elements further apart than their length."""
    t = torch.empty((case["rows"], case["d"] + case["extra"]), device="cuda", dtype=dtype)
    return t.normal_(0.0, scale, generator=gen)[:, :case["d"]]


def _gate_rows(case):
    return {"none": 0, "channel": 1, "sequence": case.get("groups", 1), "element": case["rows"]}[case["gate"]]


def _norm_inputs(case, gen):
    """The residual stream x, a block's output f, the norms' weights and the gate;
    some channels are much larger than the rest, as in trained models."""
    d, stream, branch = case["d"], KINDS[case["stream"]], KINDS[case["branch"]]
    loud = torch.where(torch.rand((d,), device="cuda", generator=gen) < 0.01, 20.0, 1.0)
    x = _rows_tensor(case, stream, gen)
    x.mul_(loud.to(stream))
    f = _rows_tensor(case, branch, gen, 0.3)
    f.add_(0.1)
    vec = lambda at, by: torch.empty((d,), device="cuda").normal_(at, by, generator=gen)  # noqa: E731
    s = {"x": x, "f": f, "post_weight": vec(1.0, 0.2), "pre_weight": vec(1.0, 0.2), "residual_scale": 0.9375}
    if case["bias"]:
        s |= {"post_bias": vec(0.0, 0.1), "pre_bias": vec(0.0, 0.1)}
    k = _gate_rows(case)
    if k:
        kind = torch.float32 if case["gate"] == "channel" else branch
        s["gate"] = torch.empty((k, d), device="cuda", dtype=kind).normal_(0.5, 0.3, generator=gen)
    return s


def _norm_saved(case, s, gen):
    """What backward has beside the forward's inputs: y, the statistics of f and y
    ([2][rows][2]: mean, reciprocal deviation), the gradients of y and h."""
    saved = _plain_forward(case, s, stats=True)
    s["y"], s["stats"] = saved["y"], saved["stats"]
    s["dy"] = _rows_tensor(case, KINDS[case["stream"]], gen, 1e-2)
    s["dh"] = _rows_tensor(case, KINDS[case["branch"]], gen, 1e-2)
    del s["x"]


def prepare(case, seed):
    gen = _generator(seed)
    if case["op"] in ("fwd", "bwd"):
        s = _norm_inputs(case, gen)
        if case["op"] == "bwd":
            _norm_saved(case, s, gen)
        return {"case": case, **s}
    places, n = _places(case)
    p, g, m, v = _adamw_inputs(case, gen, places, n)
    state = {"case": case, "params": p, "grads": g, "t": T0}
    if own:
        import paper_2510_05361_gb300 as mt
        opt = mt.AdamW(_tensors(p, places), None if g is None else _tensors(g, places), betas=BETAS, eps=EPS,
                       state_bits=case["bits"], decay=[k for _, _, k in places], seed=SEED)
        opt.t = T0
        state["optimizer"] = opt
        state["m"], state["v"] = opt.state("m"), opt.state("v")
    else:
        state["decay"] = torch.cat([torch.full((-(-k // BLOCK) * BLOCK,), c, device="cuda", dtype=torch.bfloat16)
                                    for _, k, c in places])
        state["odd"] = torch.tensor([_signed(k, 32) for k in ODD], device="cuda", dtype=torch.int32)
        make = lambda kind: {"codes": torch.empty((case["M"], n), device="cuda", dtype=kind),  # noqa: E731
                             "scales": torch.empty((case["M"], n // BLOCK), device="cuda")}
        state["m"] = make(torch.float8_e4m3fn) if case["bits"] == 8 else torch.empty_like(m)
        state["v"] = make(torch.float8_e5m2) if case["bits"] == 8 else torch.empty_like(v)
    for name, t in (("m", m), ("v", v)):
        _store(case, state[name], t, name, None)
    return state


def _tensors(flat, places):
    return [[row[at:at + k] for at, k, _ in places] for row in flat]


# ------------------------------------------------------------------ plain forms

GOLDEN = 0x9E3779B97F4A7C15
ODD = [pow(0x9E3779B1, k + 1, 1 << 32) for k in range(8)]


def _signed(k, bits):
    return k - (1 << bits) if k >= 1 << (bits - 1) else k


def _mix(z):
    """SplitMix64's output function on int64 tensors."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9, 64)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB, 64)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _key(seed, t):
    """SplitMix64's value t of the seed, as a signed number."""
    z = (seed + GOLDEN * (t + 1)) % (1 << 64)
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9 % (1 << 64)
    z = (z ^ (z >> 27)) * 0x94D049BB133111EB % (1 << 64)
    return _signed(z ^ (z >> 31), 64)


def _words(seed, t, M, n, odd):
    """Two 32-bit words an element: those of its group of eight (a counter's
    SplitMix64 value: replica and group), times an odd constant of its place."""
    counter = (torch.arange(M, device="cuda").view(M, 1) << 32) + torch.arange(n // 8, device="cuda")
    z = _mix(counter * _signed(GOLDEN, 64) + _key(seed, t))
    low, high = z.to(torch.int32), (z >> 32).to(torch.int32)
    return (low[..., None] * odd).view(M, n), (high[..., None] * odd).view(M, n)


def _moved(y, words, drop):
    """y, moved by a random part of -1/2 to 1/2 of the step between codes, given the
    bits that a code drops: the nearest code of it is y rounded stochastically."""
    by = ((words >> (32 - drop)) & ((1 << drop) - 1)) - (1 << (drop - 1))
    return torch.where(y.abs() < 2.0 ** -30, 0.0, (y.view(torch.int32) + by).view(torch.float32))


def _store(case, held, t, name, words):
    """Writes m or v as it is held: fp32, or codes with a power of two for each block."""
    if case["bits"] == 32:
        held.copy_(t)
        return
    top, drop, most = (7, 20, 448.0) if name == "m" else (14, 21, 57344.0)
    blocks = t.view(t.shape[0], -1, BLOCK)
    largest = blocks.abs().amax(2)
    power = torch.exp2(torch.floor(torch.log2(largest)))
    power = torch.where(power > largest, power * 0.5, torch.where(power * 2.0 <= largest, power * 2.0, power))
    scale = torch.where(largest < 2.0 ** -110, 0.0, power * 2.0 ** -top)
    inverse = torch.where(scale > 0.0, 1.0 / scale, 0.0)
    y = blocks * inverse[..., None]
    if name == "v":
        y = torch.where(scale[..., None] > 0.0, y.clamp(min=2.0 ** -16), y)
    y = y.view(t.shape)
    if words is not None:
        y = _moved(y, words, drop)
    held["codes"].copy_(y.clamp(-most, most).to(held["codes"].dtype))
    held["scales"].copy_(scale)


def _load(case, held):
    if case["bits"] == 32:
        return held
    codes = held["codes"]
    return (codes.float().view(codes.shape[0], -1, BLOCK) * held["scales"][..., None]).view(codes.shape)


def _plain_adamw(state, case):
    p, t = state["params"], state["t"]
    g = state["grads"].float()
    if case["clip"]:
        # the squares' sum in 64 bits: one factor that all of a replica's elements share
        norm = g.square().sum(1, keepdim=True, dtype=torch.float64).sqrt()
        g = g * torch.clamp(RHO / (norm + 1e-6), max=1.0).float()
    m = _load(case, state["m"]) * BETAS[0] + g * (1.0 - BETAS[0])
    v = _load(case, state["v"]) * BETAS[1] + g * g * (1.0 - BETAS[1])
    words = _words(SEED, t, *p.shape, state["odd"]) if case["bits"] == 8 or case["param"] == "bf16" else (None, None)
    _store(case, state["m"], m, "m", words[0])
    _store(case, state["v"], v, "v", words[1])
    root = v.sqrt_().mul_(1.0 / math.sqrt(1.0 - BETAS[1] ** (t + 1))).add_(EPS)
    x = p.float() * (1.0 - LR * DECAY * state["decay"].float()) - m.mul_(LR / (1.0 - BETAS[0] ** (t + 1))).div_(root)
    if case["param"] == "bf16":
        x = (x.view(torch.int32) + (words[0] & 0xFFFF)).bitwise_and_(-65536).view(torch.float32)
    p.copy_(x)
    state["t"] = t + 1


def _plain_average(state, case):
    p = state["params"]
    count = torch.full((), float(case["M"]), device="cuda")       # a tensor: by a number, torch would multiply by 1/M
    mean = lambda t: t.sum(0, keepdim=True).div_(count).expand(p.shape).contiguous()  # noqa: E731
    p.copy_(mean(p.float()))
    _store(case, state["m"], mean(_load(case, state["m"])), "m", None)
    _store(case, state["v"], mean(_load(case, state["v"])), "v", None)


def _gate_of(case, s):
    """The gate of every row, or 1."""
    if "gate" not in s:
        return 1.0
    gate = s["gate"].float()
    return gate.repeat_interleave(case["rows"] // gate.shape[0], 0) if gate.shape[0] not in (1, case["rows"]) else gate


def _statistics(case, z):
    """Mean (0 for "rms") and reciprocal deviation of each row."""
    mean = z.mean(1, keepdim=True) if case["norm"] == "layer" else torch.zeros_like(z[:, :1])
    return mean, torch.rsqrt((z - mean).square().mean(1, keepdim=True) + NORM_EPS)


def _plain_forward(case, s, stats=False):
    x, f = s["x"].float(), s["f"].float()
    mean_f, r_f = _statistics(case, f)
    z = (f - mean_f) * r_f * s["post_weight"] + s.get("post_bias", 0.0)
    y = s["residual_scale"] * x + _gate_of(case, s) * z
    mean_y, r_y = _statistics(case, y)
    h = (y - mean_y) * r_y * s["pre_weight"] + s.get("pre_bias", 0.0)
    out = {"y": y.to(s["x"].dtype), "h": h.to(s["f"].dtype)}
    if stats:
        out["stats"] = torch.stack([torch.cat([mean_f, r_f], 1), torch.cat([mean_y, r_y], 1)])
    return out


def _plain_norm_gradient(case, q, n, r):
    """The gradient of a norm's input, from that of its normalised output."""
    q = q - n * (q * n).mean(1, keepdim=True) - (q.mean(1, keepdim=True) if case["norm"] == "layer" else 0.0)
    return q * r


def _plain_backward(case, s):
    dh, dy, y, f = (s[k].float() for k in ("dh", "dy", "y", "f"))
    (mean_f, r_f), (mean_y, r_y) = ((k[:, :1], k[:, 1:]) for k in s["stats"])
    n_y, n_f = (y - mean_y) * r_y, (f - mean_f) * r_f
    out = {"pre_weight": (dh * n_y).sum(0)}
    total = dy + _plain_norm_gradient(case, dh * s["pre_weight"], n_y, r_y)
    out["x"] = (s["residual_scale"] * total).to(s["dy"].dtype)
    dz = total * _gate_of(case, s)
    out["post_weight"] = (dz * n_f).sum(0)
    out["f"] = _plain_norm_gradient(case, dz * s["post_weight"], n_f, r_f).to(s["dh"].dtype)
    if case["bias"]:
        out |= {"pre_bias": dh.sum(0), "post_bias": dz.sum(0)}
    if "gate" in s:
        each = total * (n_f * s["post_weight"] + s.get("post_bias", 0.0))
        out["gate"] = each.view(s["gate"].shape[0], -1, case["d"]).sum(1).to(s["gate"].dtype)
    return out


def run(state):
    case = state["case"]
    if case["op"] in ("adamw", "average"):
        if not own:
            (_plain_adamw if case["op"] == "adamw" else _plain_average)(state, case)
        elif case["op"] == "adamw":
            state["optimizer"].step(LR, weight_decay=DECAY, max_norm=RHO if case["clip"] else None)
        else:
            state["optimizer"].average()
        return {"params": state["params"], "m": state["m"], "v": state["v"]}
    if not own:
        return (_plain_forward if case["op"] == "fwd" else _plain_backward)(case, state)
    import paper_2510_05361_gb300 as mt
    if case["op"] == "fwd":
        y, h, _ = mt.peri_norm_forward(
            state["x"], state["f"], state["post_weight"], state["pre_weight"], post_bias=state.get("post_bias"),
            pre_bias=state.get("pre_bias"), gate=state.get("gate"), residual_scale=state["residual_scale"],
            eps=NORM_EPS, norm=case["norm"])
        return {"y": y, "h": h}
    return mt.peri_norm_backward(
        state["dh"], state["dy"], state["y"], state["f"], state["stats"], state["post_weight"], state["pre_weight"],
        post_bias=state.get("post_bias"), pre_bias=state.get("pre_bias"), gate=state.get("gate"),
        residual_scale=state["residual_scale"], norm=case["norm"])


# ------------------------------------------------------------------ what is asked of a pass

def work(case):
    size = lambda kind: 2 if case[kind] == "bf16" else 4  # noqa: E731
    if case["op"] in ("adamw", "average"):
        elems = case["M"] * sum(_numels(case))
        held = 2.0 * (1.0 + 4.0 / BLOCK) if case["bits"] == 8 else 8.0
        if case["op"] == "average":
            return {"bytes": elems * 2 * (size("param") + held), "flops": elems * 6}
        return {"bytes": elems * (2 * (size("param") + held) + size("grad")), "flops": elems * (18 if case["clip"] else 15)}
    elems = case["rows"] * case["d"]
    gate = 2 * size("branch") if case["gate"] == "element" else 0
    if case["op"] == "fwd":
        return {"bytes": elems * (2 * size("stream") + 2 * size("branch") + gate // 2), "flops": elems * 12}
    return {"bytes": elems * (3 * size("stream") + 3 * size("branch") + gate), "flops": elems * 30}


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    """The definitions in 64 bits.  What is held in 8 bits and the parameters in
    bf16 are given before their rounding (codes in units of their block's scale)."""
    gen = _generator(seed)
    if case["op"] in ("fwd", "bwd"):
        s = _norm_inputs(case, gen)
        if case["op"] == "bwd":
            _norm_saved(case, s, gen)
        return _exact_norm(case, s)
    places, n = _places(case)
    p, g, m, v = _adamw_inputs(case, gen, places, n)
    held = []
    for name, t in (("m", m), ("v", v)):
        if case["bits"] == 8:
            kind = torch.float8_e4m3fn if name == "m" else torch.float8_e5m2
            codes = {"codes": torch.empty(t.shape, device="cuda", dtype=kind),
                     "scales": torch.empty((t.shape[0], n // BLOCK), device="cuda")}
            _store(case, codes, t, name, None)
            t = codes["codes"].double().view(t.shape[0], -1, BLOCK).mul_(codes["scales"].double()[..., None])
        held.append(t.view(p.shape).double())
    m, v = held
    x = p.double()
    if case["op"] == "average":
        count = torch.full((), float(case["M"]), dtype=torch.float64, device="cuda")
        x, m, v = ((t.sum(0, keepdim=True) / count).repeat(case["M"], 1) for t in (x, m, v))
    else:
        t = T0 + 1
        u = g.double()
        if case["clip"]:
            u = u * torch.minimum(RHO / (torch.linalg.vector_norm(u, dim=1, keepdim=True) + 1e-6),
                                  torch.ones((), dtype=torch.float64, device="cuda"))
        m.lerp_(u, 1.0 - BETAS[0])
        v.lerp_(u.square_(), 1.0 - BETAS[1])
        for at, k, c in places:
            part = slice(at, at + k)
            step = m[:, part] / (1.0 - BETAS[0] ** t) / (torch.sqrt(v[:, part] / (1.0 - BETAS[1] ** t)) + EPS)
            x[:, part] = (1.0 - LR * DECAY * c) * x[:, part] - LR * step
    if case["bits"] == 32:
        return {"params": x, "m": m, "v": v}
    return {"params": x, "m": _exact_held(m, 7, 0.0), "v": _exact_held(v, 14, 2.0 ** -16)}


def _exact_held(t, top, least):
    blocks = t.view(t.shape[0], -1, BLOCK)
    largest = blocks.abs().amax(2)
    scale = torch.where(largest > 0, torch.ldexp(torch.ones_like(largest), torch.frexp(largest).exponent - 1 - top), 0.0)
    codes = torch.where(scale[..., None] > 0, blocks / scale[..., None], 0.0)
    if least:
        codes = torch.where(scale[..., None] > 0, codes.clamp(min=least), codes)
    return {"codes": codes.view(t.shape), "scales": scale}


def _exact_norm(case, s):
    s = {k: a.double() if isinstance(a, torch.Tensor) else a for k, a in s.items()}
    rows, d = case["rows"], case["d"]
    gate = torch.ones((1, d), dtype=torch.float64, device="cuda") if "gate" not in s else s["gate"]
    per = rows // gate.shape[0]
    w_post, w_pre = s["post_weight"], s["pre_weight"]
    zero = torch.zeros((d,), dtype=torch.float64, device="cuda")
    b_post, b_pre = s.get("post_bias", zero), s.get("pre_bias", zero)
    layer = case["norm"] == "layer"

    def norm(z):
        if layer:
            z = z - torch.sum(z, 1, keepdim=True) / d
        return z / torch.sqrt(torch.sum(z * z, 1, keepdim=True) / d + NORM_EPS)

    if case["op"] == "fwd":
        z = (norm(s["f"]) * w_post + b_post).view(gate.shape[0], per, d) * gate[:, None]
        y = s["residual_scale"] * s["x"] + z.view(rows, d)
        return {"y": y, "h": norm(y) * w_pre + b_pre}

    def through(q, n, r):
        back = q - n * (torch.sum(q * n, 1, keepdim=True) / d)
        if layer:
            back = back - torch.sum(q, 1, keepdim=True) / d
        return back * r

    stats = s["stats"]
    r_f, r_y = stats[0, :, 1:], stats[1, :, 1:]
    n_f, n_y = (s["f"] - stats[0, :, :1]) * r_f, (s["y"] - stats[1, :, :1]) * r_y
    dY = s["dy"] + through(s["dh"] * w_pre, n_y, r_y)
    dz = (dY.view(gate.shape[0], per, d) * gate[:, None]).view(rows, d)
    out = {"x": s["residual_scale"] * dY, "f": through(dz * w_post, n_f, r_f),
           "pre_weight": torch.einsum("rd,rd->d", s["dh"], n_y), "post_weight": torch.einsum("rd,rd->d", dz, n_f)}
    if case["bias"]:
        out |= {"pre_bias": s["dh"].sum(0), "post_bias": dz.sum(0)}
    if "gate" in s:
        out["gate"] = (dY * (n_f * w_post + b_post)).view(gate.shape[0], per, d).sum(1)
    return out
