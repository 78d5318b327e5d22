"""What is timed of the operators that train a decoder layer's gated feed-forward block and step its weights.

Three operators, each through its public entry points, beside a plain form in elementary tensor operations: the gated
feed-forward block (two projections, the activation of one times the other, the projection back; training with its backward
pass, prompts, few tokens at a time), and the AdamW step over many tensors at once with its states in 32 or in 8 bits, behind
the squared norm of all gradients that it clips by.  Widths are those of the named workloads (``inputs.WORKLOADS``), of the
tests, or generic ones.
"""
import math

import torch

own = False   # true: the library's kernels, false: the plain form

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 256           # elements that share the scale of an 8-bit state
E4M3_MOST = 448.0
BETA1, BETA2, EPS, DECAY = 0.9, 0.95, 1e-8, 0.1


# ------------------------------------------------------------------ the cases
def _text(numbers):
    return ",".join(str(n) for n in numbers)


def _numbers(text):
    return [int(n) for n in text.split(",")]


def _gated(name, tokens, hidden, ffn, gate, dtype="bf16", backward=True):
    """backward: a training step (the pre-activations are kept, all gradients come out), else the forward pass of a model in use."""
    return {"name": name, "kind": "gated", "tokens": tokens, "hidden": hidden, "ffn": ffn, "gate": gate, "dtype": dtype, "backward": backward}


def _adam(name, counts, bits, grads, step, clip=1.0, lr=2e-5):
    """counts: elements of the tensors, every second of which decays; bits: of the states; grads: type of the gradients; clip: 0 for none."""
    return {"name": name, "kind": "adam", "counts": _text(counts), "bits": bits, "grads": grads, "step": step, "clip": clip, "lr": lr}


def _layer(hidden, ffn):
    """Elements of a decoder layer's parameters: two norms, q, k and v of 4 heads of keys, the projection, the gated block."""
    return [hidden, hidden * (hidden + 2 * 512), hidden * hidden, hidden, 2 * ffn * hidden, hidden * ffn]


def listed():
    gains = [1, 2048, 7, 520, 64, 129, 1000, 4096, 31, 256, 255, 257, 2560, 640, 96, 3, 777, 1536, 2048, 12, 4095, 330, 8, 1024, 63, 20480]
    odd = [61 * 520, 5, 8191 * 33, 4097, 1, 1000 * 77, 12345, 999 * 999, 255, 65536, 3 * 257, 2500 * 130, 40 * 41, 17, 701 * 512, 100003]
    return [
        # the smallest call of a model in use: one sequence's next token, where the weights' way from memory is all
        _gated("one_token", 1, 2048, 8192, "silu", backward=False),
        # ... of a batch of sequences, at the MT-NLG slice's widths
        _gated("single_tokens", 24, 20480, 10240, "gelu_tanh", backward=False),
        # a prompt of an odd length, at a width that no tile divides
        _gated("prompt", 777, 2048, 5464, "silu", backward=False),
        # ordinary training: 4 x 2048 tokens at the 1.3B shape's widths
        _gated("training", 8192, 2048, 8192, "silu"),
        # the largest: the MT-NLG slice's widths
        _gated("training_mtnlg", 2048, 20480, 10240, "gelu_tanh"),
        # the smallest training call: somebody debugs or verifies in fp32, odd sizes
        _gated("training_small", 61, 520, 344, "gelu_erf", "fp32"),
        # the smallest step: gains and biases, where launches and latency count
        _adam("gains", gains, 32, "fp32", 3),
        # ordinary training: two layers at the 1.3B shape's widths, everything in fp32
        _adam("layers", _layer(2048, 8192) * 2, 32, "fp32", 1000),
        # four such layers with states in 8 bits and gradients in bf16
        _adam("layers_e4m3", _layer(2048, 8192) * 4, 8, "bf16", 1000),
        # many tensors of odd sizes, 8 bits, not clipped
        _adam("odd_e4m3", odd * 7, 8, "fp32", 20, clip=0.0),
    ]


def _log_int(rng, lo, hi, step=1):
    """Spread evenly over the logarithm, a multiple of ``step``."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    while True:
        if rng.random() < 0.6:
            what = rng.choice(["train", "train", "fp32", "prompt", "few", "few"])
            tokens = _log_int(rng, 1, 64) if what == "few" else _log_int(rng, 16, 1024 if what == "fp32" else 8192)
            dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"]) if what in ("few", "prompt") else "fp32" if what == "fp32" else "bf16"
            c = _gated("drawn", tokens, _log_int(rng, 64, 8192, 8), _log_int(rng, 64, 11264, 8), rng.choice(["silu", "silu", "gelu_tanh", "gelu_erf"]),
                       dtype, what in ("train", "fp32"))
            limit = 1.5e11 if dtype == "fp32" else 4.0e12
        else:
            most = _log_int(rng, 100, 2 * 8192 * 2048)
            counts = [_log_int(rng, rng.choice([1, max(1, most // 50)]), most) for _ in range(_log_int(rng, 1, 200))]
            c = _adam("drawn", counts, rng.choice([8, 8, 32]), rng.choice(["fp32", "bf16"]), _log_int(rng, 1, 100000),
                      rng.choice([0.0, 1.0, 1.0]), rng.choice([3e-6, 1e-5, 2e-5]))
            limit = math.inf
        c.pop("name")
        w = work(c)
        if w["flops"] <= limit and w["bytes"] <= 4.0e9:
            return c


# ------------------------------------------------------------------ what a program has in hand
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, g, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _gated_state(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    t, h, f = c["tokens"], c["hidden"], c["ffn"]
    new = lambda *shape: torch.empty(shape, dtype=dt, device="cuda")   # noqa: E731
    s = {"x": _randn((t, h), g, dt), "w_fc1": _randn((2 * f, h), g, dt, 1.0 / math.sqrt(h)), "w_fc2": _randn((h, f), g, dt, 1.0 / math.sqrt(f)),
         "g": new(t, f), "y": new(t, h)}
    if c["backward"]:
        s.update(dy=_randn((t, h), g, dt), z=new(t, 2 * f), dz=new(t, 2 * f), dx=new(t, h), dw_fc1=new(2 * f, h), dw_fc2=new(h, f))
    return s


def _places(counts):
    """Where each tensor begins in a buffer of all of them, at whole blocks, and the buffer's length."""
    at, out = 0, []
    for n in counts:
        out.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return out, at


def _to_e4m3(x):
    """Codes and scales of a buffer of whole blocks, to nearest (the states that a program comes with)."""
    most = x.view(-1, BLOCK).abs().amax(1)
    scale = torch.where(most > 0, most / E4M3_MOST, 1.0)
    return (x.view(-1, BLOCK) / scale[:, None]).clamp_(-E4M3_MOST, E4M3_MOST).view(-1).to(torch.float8_e4m3fn), scale


def _adam_state(c, seed):
    g, counts = _gen(seed), _numbers(c["counts"])
    places, total = _places(counts)
    # zeros between the tensors; parts of a model have gradients of different sizes, by row and by tensor
    blocks = torch.tensor([n // BLOCK for n in counts], device="cuda")
    rest = torch.tensor([n % BLOCK for n in counts], device="cuda")
    first = torch.tensor([p // BLOCK for p in places], device="cuda")
    inside = torch.ones((total // BLOCK, BLOCK), dtype=torch.bool, device="cuda")
    short = rest > 0
    inside[(first + blocks)[short]] = torch.arange(BLOCK, device="cuda") < rest[short][:, None]
    inside = inside.view(-1)
    sizes = torch.exp(0.7 * torch.randn((total // BLOCK, 1), generator=g, device="cuda"))
    flat = lambda scale: ((torch.randn((total // BLOCK, BLOCK), generator=g, device="cuda") * sizes).view(-1) * scale) * inside   # noqa: E731
    grad = flat(1e-4)
    m, root = flat(4e-5), flat(1e-4).abs() + 3e-5 * inside
    s = {"master": _randn((total,), g, scale=0.02) * inside, "grad": grad.to(DTYPES[c["grads"]]),
         "weight": torch.zeros(total, dtype=torch.bfloat16, device="cuda"), "sqnorm": torch.zeros(1, device="cuda"), "places": places, "counts": counts,
         "seed": seed * 7919 + 13}
    if c["bits"] == 8:
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _to_e4m3(m), _to_e4m3(root)
    else:
        s["m"], s["v"] = m, root.square()
    s["decay"] = torch.repeat_interleave(torch.arange(len(counts), device="cuda") % 2, torch.tensor([(n + BLOCK - 1) // BLOCK for n in counts], device="cuda"),
                                         output_size=total // BLOCK)
    return s


def prepare(case, seed):
    s = {"gated": _gated_state, "adam": _adam_state}[case["kind"]](case, seed)
    s["case"] = case
    return s


# ------------------------------------------------------------------ the plain forms
def _act(kind, x):
    """The activation and its derivative."""
    if kind == "silu":
        sig = torch.sigmoid(x)
        return x * sig, sig * (1 + x * (1 - sig))
    if kind == "gelu_erf":
        cdf = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * cdf, cdf + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (x + 0.044715 * x * x * x))
    return 0.5 * x * (1 + th), 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * k * (1 + 3 * 0.044715 * x * x)


def _plain_gated(c, s):
    f = c["ffn"]
    w1, w2, x = s["w_fc1"].float(), s["w_fc2"].float(), s["x"].float()
    z = x @ w1.T
    s["g"].copy_(_act(c["gate"], z[:, :f])[0] * z[:, f:])
    g = s["g"].float()   # what is stored is what the next product takes, and what the backward pass reads
    s["y"].copy_(g @ w2.T)
    if c["backward"]:
        s["z"].copy_(z)
        dy, z = s["dy"].float(), s["z"].float()
        a, da = _act(c["gate"], z[:, :f])
        dg = dy @ w2
        s["dz"][:, :f] = dg * z[:, f:] * da
        s["dz"][:, f:] = dg * a
        dz = s["dz"].float()
        s["dx"].copy_(dz @ w1)
        s["dw_fc1"].copy_(dz.T @ x)
        s["dw_fc2"].copy_(dy.T @ g)


LOW = 0xFFFFFFFF


def _keys(seed, step):
    """Two words of 32 bits of a step's random numbers."""
    whole = (1 << 64) - 1
    s = (seed * 0x9E3779B97F4A7C15 + step) & whole
    s = ((s ^ (s >> 32)) * 0xBB67AE8584CAA73B) & whole
    s = ((s ^ (s >> 29)) * 0x6A09E667F3BCC909) & whole
    s ^= s >> 32
    return s & LOW, s >> 32


def _random(s, c):
    """Numbers in (0, 1) for the rounding of each element's m and v: integer arithmetic on the step's seed, the number of the block among
    all tensors' and the element's place in it."""
    lo, hi = _keys(s["seed"], c["step"])
    signed = lambda x: x - (1 << 64) if x >= 1 << 63 else x   # noqa: E731
    times = lambda x, by: (x * signed(by)) & LOW   # noqa: E731
    b = torch.arange(s["master"].numel() // BLOCK, device="cuda")
    k = (times(b, 0x9E3779B1) + lo) & LOW
    k = times(k ^ (k >> 15), 0x510E527F)
    k = (k ^ (k >> 13)) ^ hi
    h = (k[:, None] + times(torch.arange(BLOCK, device="cuda"), 0x3C6EF373)) & LOW
    h = times(h ^ (h >> 16), 0x6A09E667)
    h = times(h ^ (h >> 15), 0xBB67AE85)
    h = (h ^ (h >> 16)).view(-1)
    return ((h & 0xFFFF).double() + 0.5) / 65536, ((h >> 16).double() + 0.5) / 65536


def _rounded(x, u, least):
    """A buffer in 8 bits, rounded up where the part of a step that is left and u make a whole one; codes of what is not zero are at
    least ``least`` steps."""
    most = x.view(-1, BLOCK).abs().amax(1)
    scale = torch.where(most > 0, (most / E4M3_MOST).clamp_(min=2.0 ** -126), 1.0)
    y = (x.view(-1, BLOCK).abs() * (1.0 / scale)[:, None]).clamp_(max=E4M3_MOST).view(-1)
    step = torch.ldexp(torch.ones((), device="cuda"), (torch.frexp(y).exponent - 1).clamp_(min=-6) - 3)
    k = (y.double() / step + u).floor_()
    k = torch.where(x != 0, k.clamp_(min=least), 0.0)
    return torch.copysign(k * step, x.double()).float().to(torch.float8_e4m3fn), scale


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _plain_adam(c, s):
    total = s["master"].numel()
    s["sqnorm"][0] = s["grad"].double().square().sum()   # a long sum
    g = s["grad"].float()
    if c["clip"] > 0:
        g = g * torch.clamp(_f32(c["clip"]) / (s["sqnorm"].sqrt() + 1e-6), max=1.0)
    blocks = lambda codes, scale: (codes.float().view(-1, BLOCK) * scale[:, None]).view(-1)   # noqa: E731
    if c["bits"] == 8:
        m, v = blocks(s["m"], s["m_scale"]), blocks(s["v"], s["v_scale"]).square()
    else:
        m, v = s["m"], s["v"]
    b1, b2 = _f32(BETA1), _f32(BETA2)
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * (1 - b2) * g
    p = s["master"]
    update = m / (1 - b1 ** c["step"]) / ((v / (1 - b2 ** c["step"])).sqrt() + _f32(EPS))
    decays = _f32(DECAY) * s["decay"].float().repeat_interleave(BLOCK, output_size=total)
    p.sub_((update + decays * p) * _f32(c["lr"]))
    s["weight"].copy_(p)
    if c["bits"] == 8:
        um, uv = _random(s, c)
        for k, x, u, least in (("m", m, um, 0), ("v", v.sqrt(), uv, 1)):
            codes, scale = _rounded(x, u, least)
            s[k].copy_(codes)
            s[k + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


# ------------------------------------------------------------------ one pass
def _own_gated(c, s):
    import paper_2201_11990_amd as M
    gate = {"silu": M.GATE_SILU, "gelu_tanh": M.GATE_GELU_TANH, "gelu_erf": M.GATE_GELU_ERF}[c["gate"]]
    desc = M.gated_desc(s["x"], s["w_fc1"], gate)
    if "workspace" not in s:   # kept from step to step, as a training program or a server does
        s["workspace"] = torch.empty(max(16, M.mtnlg_gated_ffn_workspace(desc)), dtype=torch.uint8, device="cuda")
    M.mtnlg_gated_ffn_fwd(desc, s["x"], s["w_fc1"], s["w_fc2"], s.get("z"), s["g"], s["y"], s["workspace"])
    if c["backward"]:
        M.mtnlg_gated_ffn_bwd(desc, s["x"], s["w_fc1"], s["w_fc2"], s["z"], s["g"], s["dy"], s["dz"], s["dx"], s["dw_fc1"], s["dw_fc2"], s["workspace"])


def _own_adam(c, s):
    import paper_2201_11990_amd as M
    if "tensors" not in s:   # a training program's buffers stay where they are
        part = lambda k, a, n: s[k][a:a + n]   # noqa: E731
        rows = []
        for i, (a, n) in enumerate(zip(s["places"], s["counts"])):
            row = {"master": part("master", a, n), "m": part("m", a, n), "v": part("v", a, n), "grad": part("grad", a, n),
                   "weight_bf16": part("weight", a, n), "decay": i % 2 == 1}
            if c["bits"] == 8:
                row.update(m_scale=part("m_scale", a // BLOCK, -(-n // BLOCK)), v_scale=part("v_scale", a // BLOCK, -(-n // BLOCK)))
            rows.append(row)
        s["tensors"] = M.AdamTensors(rows)
        s["workspace"] = torch.empty(M.mtnlg_grad_sqnorm_many_workspace(), dtype=torch.uint8, device="cuda")
    M.mtnlg_grad_sqnorm_many(s["tensors"], s["sqnorm"], s["workspace"])
    M.mtnlg_adam_step_many(s["tensors"], s["sqnorm"], lr=c["lr"], step=c["step"], beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                           max_grad_norm=c["clip"], seed=s["seed"])


def _results(c):
    if c["kind"] == "gated":
        return ("g", "y", "z", "dz", "dx", "dw_fc1", "dw_fc2") if c["backward"] else ("g", "y")
    return ("sqnorm", "master", "weight", "m", "v") + (("m_scale", "v_scale") if c["bits"] == 8 else ())


def run(state):
    c = state["case"]
    if own:
        {"gated": _own_gated, "adam": _own_adam}[c["kind"]](c, state)
    else:
        {"gated": _plain_gated, "adam": _plain_adam}[c["kind"]](c, state)
    return {k: state[k] for k in _results(c)}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "gated":
        t, h, f, es = c["tokens"], c["hidden"], c["ffn"], 2 if c["dtype"] == "bf16" else 4
        w = 3 * h * f
        forward = es * (w + t * (2 * h + f))   # x and the weights in, g and y out
        if not c["backward"]:
            return {"bytes": forward, "flops": 2.0 * t * w}
        # z out too; backward: x, z, g, dy and the weights in, dz, dx and the weights' gradients out
        backward = es * (2 * w + t * (3 * h + 5 * f))
        return {"bytes": forward + es * t * 2 * f + backward, "flops": 6.0 * t * w}
    n = sum(_numbers(c["counts"]))
    grads = 4 if c["grads"] == "fp32" else 2
    # the norm reads the gradients; the step reads them and weight, m, v, and writes weight, its rounded copy, m, v
    state = 2.0 + 8.0 / BLOCK if c["bits"] == 8 else 8.0
    return {"bytes": n * (2 * grads + 4 + 4 + 2 + 2 * state), "flops": 18.0 * n}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_act(kind, x):
    x = x.detach().requires_grad_()
    y = {"silu": torch.nn.functional.silu, "gelu_erf": torch.nn.functional.gelu, "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[kind](x)
    (slope,) = torch.autograd.grad(y.sum(), x)
    return y.detach(), slope


def _exact_gated(c, s):
    dt, f = DTYPES[c["dtype"]], c["ffn"]
    stored = lambda t: t.to(dt).double()   # noqa: E731
    x, w1, w2 = s["x"].double(), s["w_fc1"].double(), s["w_fc2"].double()
    up, gate = x @ w1[f:].T, x @ w1[:f].T
    out = {"g": _exact_act(c["gate"], gate)[0] * up}
    g = stored(out["g"])
    out["y"] = g @ w2.T
    if c["backward"]:
        out["z"] = torch.cat([gate, up], 1)
        gate, up, dy = stored(gate), stored(up), s["dy"].double()
        act, slope = _exact_act(c["gate"], gate)
        dg = dy @ w2
        out["dz"] = torch.cat([dg * up * slope, dg * act], 1)
        dz = stored(out["dz"])
        out["dx"] = dz[:, :f] @ w1[:f] + dz[:, f:] @ w1[f:]
        out["dw_fc1"] = dz.T @ x
        out["dw_fc2"] = dy.T @ g
    return out


def _exact_codes(x, u, least):
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1) / E4M3_MOST
    scale = torch.where(scale > 0, scale.clamp(min=2.0 ** -126), 1.0)
    y = (x.abs() / scale[:, None]).clamp(max=E4M3_MOST)
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    low = torch.floor(y / step)
    k = low + ((y / step - low) >= 1 - u.view(-1, BLOCK))
    k = torch.where((x != 0) & (k < least), float(least), k)
    return (torch.sign(x) * k * step).view(-1), scale


def _exact_adam(c, s):
    blocks = lambda codes, scale: (codes.float().double().view(-1, BLOCK) * scale.double()[:, None]).view(-1)   # noqa: E731
    g, p = s["grad"].double(), s["master"].double()
    sqnorm = torch.dot(g, g)
    if c["clip"] > 0:
        g = g * min(1.0, c["clip"] / (math.sqrt(float(sqnorm)) + 1e-6))
    m, v = (blocks(s["m"], s["m_scale"]), blocks(s["v"], s["v_scale"]) ** 2) if c["bits"] == 8 else (s["m"].double(), s["v"].double())
    b1, b2 = _f32(BETA1), _f32(BETA2)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    decays = (_f32(DECAY) * s["decay"].double()).view(-1, 1)
    update = (m / (1 - b1 ** c["step"])) / (torch.sqrt(v / (1 - b2 ** c["step"])) + _f32(EPS))
    p = p - _f32(c["lr"]) * (update + (decays * p.view(-1, BLOCK)).view(-1))
    out = {"sqnorm": sqnorm.view(1), "master": p, "weight": p}
    if c["bits"] == 8:
        um, uv = _random(s, c)
        (out["m"], out["m_scale"]), (out["v"], out["v_scale"]) = _exact_codes(m, um, 0), _exact_codes(torch.sqrt(v), uv, 1)
    else:
        out.update(m=m, v=v)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _exact_gated, "adam": _exact_adam}[case["kind"]](case, s)
