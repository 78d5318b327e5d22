"""What is timed of the operators for decoder layers with rotary positions, RMS norms and grouped heads on packed batches.

Three operators, each through its public entry points, beside a plain form in elementary tensor operations: causal attention
over packed sequences of different lengths with grouped heads (forward and backward, whole prompts, prompts continued on a
cache, single tokens), rotary positions (forward and backward), and the root-mean-square norm with the residual's addition
(forward and backward, and with its result in 8 bits).  Head sizes and widths are those of the named workloads
(``inputs.WORKLOADS``), of the tests, or generic ones.
"""
import math

import torch

own = False   # true: the library's kernels, false: the plain form

EPS = 1e-5
BASE = 10000.0
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
E4M3_MOST = 448.0


# ------------------------------------------------------------------ the cases
def _text(lengths):
    return ",".join(str(n) for n in lengths)


def _lengths(text):
    return [int(n) for n in text.split(",")]


def _attention(name, queries, keys, kv_heads, group, head_dim, dtype="bf16", backward=True, fused=False, cache=False):
    """queries, keys: lengths of the sequences; group: query heads to a head of keys; fused: q, k and v are parts of one
    matrix [token][kv head][q .. q k v]; cache: keys lie in regions that are longer than what is filled."""
    return {"name": name, "kind": "attention", "queries": _text(queries), "keys": _text(keys), "kv_heads": kv_heads, "group": group,
            "head_dim": head_dim, "dtype": dtype, "backward": backward, "fused": fused, "cache": cache}


def _rotary(name, tokens, kv_heads, group, head_dim, rotary_dim, layout, scaling, dtype="bf16"):
    return {"name": name, "kind": "rotary", "tokens": tokens, "kv_heads": kv_heads, "group": group, "head_dim": head_dim,
            "rotary_dim": rotary_dim, "layout": layout, "scaling": scaling, "dtype": dtype}


def _rmsnorm(name, tokens, hidden, dtype="bf16", backward=True, columns=None):
    """columns: the result goes out in 8 bits, a scale to so many columns (0: to the row); None: in the inputs' type."""
    return {"name": name, "kind": "rmsnorm", "tokens": tokens, "hidden": hidden, "dtype": dtype, "backward": backward,
            "eight_bits": columns is not None, "columns": columns or 0}


def listed():
    one_each = [5907, 311, 13121, 1024, 887, 2450, 76, 9001, 1601, 640, 4096, 230, 3333, 1500, 702, 7168,
                129, 2047, 512, 3801, 15872, 96, 1130, 6007, 411, 2900, 820, 5200, 1984, 333, 10240, 64]
    return [
        # the smallest call: a few short documents and an empty place of the batch, where launches and latency count
        _attention("packed_small", [17, 0, 64, 130], [17, 0, 64, 130], 2, 2, 64),
        # ordinary training: documents of many lengths packed into a micro-batch of 4 x 2048 tokens, the 1.3B shape's heads
        _attention("packed_documents", [1213, 402, 2048, 77, 960, 1511, 333, 1648], [1213, 402, 2048, 77, 960, 1511, 333, 1648], 4, 4, 128,
                   fused=True),
        # two long documents of odd lengths, the MT-NLG slice's head size, all 16 heads with keys of their own
        _attention("packed_d160", [2501, 1589], [2501, 1589], 16, 1, 160),
        # the largest: long-context training, one document much longer than the others
        _attention("packed_long", [9001, 4990, 2009, 384], [9001, 4990, 2009, 384], 8, 4, 128),
        # fp32: somebody verifies or trains a small model; a head size between the usual ones
        _attention("packed_fp32", [700, 129, 451, 256], [700, 129, 451, 256], 4, 2, 96, "fp32"),
        # a model in use: prompts continued in pieces, behind what the cache holds already
        _attention("prompts_continued", [512, 384, 77], [4608, 1500, 77], 8, 4, 128, backward=False),
        # ... and single tokens of many sequences over their caches
        _attention("single_tokens", [1] * len(one_each), one_each, 8, 4, 128, backward=False, cache=True),
        # rotary positions of queries and keys for long contexts, in training: forward and its gradient
        _rotary("rotary_documents", 8192, 4, 4, 128, 128, "half", "parts"),
        # the smallest: a quarter of the head turns, pairs side by side, fp32
        _rotary("rotary_small", 230, 2, 2, 64, 16, "interleaved", "none", "fp32"),
        # one norm of the MT-NLG slice with the residual before it, forward and backward
        _rmsnorm("rmsnorm_mtnlg", 2048, 20480),
        # ... whose result the next product takes in 8 bits
        _rmsnorm("rmsnorm_e4m3", 8192, 2048, backward=False, columns=128),
        # the smallest: a debugging run
        _rmsnorm("rmsnorm_small", 61, 520, "fp32"),
    ]


def _log_int(rng, lo, hi, step=1):
    """Spread evenly over the logarithm, a multiple of ``step``."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def _draw_attention(rng):
    what = rng.choice(["train", "train", "train", "fp32", "continued", "single"])
    d = rng.choice([64, 128, 128, 160, 8 * rng.randint(4, 24), 256])
    kv, group = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([1, 1, 2, 3, 4, 7, 8])
    if what in ("train", "fp32"):
        count, most = _log_int(rng, 1, 48), _log_int(rng, 16, 8192 if what == "train" else 1024)
        least = rng.choice([1, max(1, most // 10)])
        lengths = [_log_int(rng, least, most) if rng.random() < 0.95 else 0 for _ in range(count)]
        if sum(lengths) == 0:
            lengths[0] = most
        return _attention("drawn", lengths, lengths, kv, group, d, "bf16" if what == "train" else "fp32", fused=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if what == "continued":
        queries = [_log_int(rng, rng.choice([1, 64]), 1024) for _ in range(_log_int(rng, 1, 16))]
        return _attention("drawn", queries, [n + rng.choice([0, _log_int(rng, 1, 8192)]) for n in queries], kv, group, d, dtype, backward=False,
                          cache=rng.random() < 0.5)
    keys = [_log_int(rng, rng.choice([1, 256]), 16384) for _ in range(_log_int(rng, 1, 64))]
    return _attention("drawn", [1] * len(keys), keys, kv, group, d, dtype, backward=False, cache=True)


def draw(rng):
    while True:
        kind = rng.choice(["attention"] * 4 + ["rotary", "rmsnorm", "rmsnorm"])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        if kind == "attention":
            c = _draw_attention(rng)
        elif kind == "rotary":
            d = 8 * rng.randint(4, 32)
            c = _rotary("drawn", _log_int(rng, 1, 8192), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8]), d,
                        rng.choice([d, 16 * rng.randint(1, d // 16)]), rng.choice(["half", "interleaved"]),
                        rng.choice(["none", "linear", "base", "parts"]), dtype)
        else:
            c = _rmsnorm("drawn", _log_int(rng, 1, 8192), _log_int(rng, 64, 20480, 8), dtype, True)
            if rng.random() < 0.4:
                c = _rmsnorm("drawn", c["tokens"], c["hidden"], dtype, False, rng.choice([0, 128]))
        c.pop("name")
        w = work(c)
        limit = 2.0e11 if c["dtype"] == "fp32" else 3.0e12
        pairs = max([0] + [a * b for a, b in zip(_lengths(c["queries"]), _lengths(c["keys"]))]) * c["kv_heads"] * c["group"] if kind == "attention" else 0
        if w["flops"] <= limit and w["bytes"] <= 1.0e9 and pairs <= 2.6e9:
            return c


# ------------------------------------------------------------------ what a program has in hand
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, g, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _attention_state(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    ql, kl = _lengths(c["queries"]), _lengths(c["keys"])
    kv, r, d = c["kv_heads"], c["group"], c["head_dim"]
    regions = [(n + 255) // 256 * 256 for n in kl] if c["cache"] else kl
    q_off, k_off = _offsets(ql), _offsets(regions)
    tq, tk = q_off[-1], k_off[-1]
    if c["fused"]:   # one projection's result
        qkv = _randn((tq, kv, r + 2, d), g, dt)
        grad = torch.empty_like(qkv)
        parts = lambda t: (t[:, :, :r], t[:, :, r], t[:, :, r + 1])   # noqa: E731
        (q, k, v), (dq, dk, dv) = parts(qkv), parts(grad)
    else:
        q, k, v = _randn((tq, kv, r, d), g, dt), _randn((tk, kv, d), g, dt), _randn((tk, kv, d), g, dt)
        dq, dk, dv = (torch.empty_like(t) for t in (q, k, v)) if c["backward"] else (None, None, None)
    int32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    s = {"q": q, "k": k, "v": v, "a": torch.empty((tq, kv, r, d), dtype=dt, device="cuda"), "lse": torch.empty((kv * r, tq), device="cuda"),
         "q_offsets": int32(q_off), "k_offsets": int32(k_off), "k_lengths": int32(kl) if c["cache"] else None,
         "max_q": max(ql), "max_k": max(kl), "host": (ql, kl, q_off, k_off)}
    if c["backward"]:
        s.update(da=_randn((tq, kv, r, d), g, dt), dq=dq, dk=dk, dv=dv)
    return s


def _rotary_state(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    t, kv, r, d = c["tokens"], c["kv_heads"], c["group"], c["head_dim"]
    # documents that start anywhere in a batch of long contexts: positions run up, and begin again a few times
    begin = torch.randint(0, max(1, t // 3 + 1), (t,), generator=g, device="cuda") == 0
    start = torch.where(begin, torch.arange(t, device="cuda"), 0).cummax(0).values
    far = int(torch.randint(0, 30000, (1,), generator=g, device="cuda"))
    s = {"q": _randn((t, kv, r, d), g, dt), "k": _randn((t, kv, d), g, dt), "dq_out": _randn((t, kv, r, d), g, dt),
         "dk_out": _randn((t, kv, d), g, dt), "positions": (torch.arange(t, device="cuda") - start + far).to(torch.int32)}
    for name, like in (("q_out", "q"), ("k_out", "k"), ("dq", "q"), ("dk", "k")):
        s[name] = torch.empty_like(s[like])
    return s


def _rmsnorm_state(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    t, h = c["tokens"], c["hidden"]
    s = {"x": _randn((t, h), g, dt), "residual": _randn((t, h), g, dt, 3.0), "gamma": _randn((h,), g, dt, 0.1) + 1,
         "xsum": torch.empty((t, h), dtype=dt, device="cuda"), "rstd": torch.empty(t, device="cuda")}
    if c["eight_bits"]:
        s.update(out=torch.empty((t, h), dtype=torch.float8_e4m3fn, device="cuda"),
                 scale=torch.empty((t, -(-h // (c["columns"] or h))), device="cuda"))
    else:
        s["out"] = torch.empty((t, h), dtype=dt, device="cuda")
    if c["backward"]:
        s.update(dout=_randn((t, h), g, dt), dres=_randn((t, h), g, dt), dx=torch.empty((t, h), dtype=dt, device="cuda"),
                 dgamma=torch.empty(h, device="cuda"))
    return s


def prepare(case, seed):
    s = {"attention": _attention_state, "rotary": _rotary_state, "rmsnorm": _rmsnorm_state}[case["kind"]](case, seed)
    s["case"] = case
    return s


# ------------------------------------------------------------------ the plain forms
def _plain_attention(c, s):
    ql, kl, q_off, k_off = s["host"]
    kv, r, d = c["kv_heads"], c["group"], c["head_dim"]
    scale = 1.0 / math.sqrt(d)
    for lq, lk, q0, k0 in zip(ql, kl, q_off, k_off):   # sequences of a packed batch see nothing of each other
        if lq == 0:
            continue
        rows = lambda t: t[q0:q0 + lq].permute(1, 2, 0, 3).reshape(kv, r * lq, d).float()   # noqa: E731
        keys = lambda t: t[k0:k0 + lk].transpose(0, 1).float()   # noqa: E731
        q, k, v = rows(s["q"]), keys(s["k"]), keys(s["v"])
        hidden = torch.arange(lk, device="cuda") > torch.arange(lq, device="cuda")[:, None] + (lk - lq)
        p = (q @ k.transpose(1, 2)).mul_(scale).view(kv, r, lq, lk).masked_fill_(hidden, -math.inf)
        most = p.amax(-1, keepdim=True)
        p = p.sub_(most).exp_()
        total = p.sum(-1, keepdim=True)
        p = p.div_(total).view(kv, r * lq, lk)
        a = p @ v
        back = lambda t: t.view(kv, r, lq, d).permute(2, 0, 1, 3)   # noqa: E731
        s["a"][q0:q0 + lq] = back(a)
        s["lse"][:, q0:q0 + lq] = (most + total.log()).view(kv * r, lq)
        if c["backward"]:
            da = rows(s["da"])
            ds = (da @ v.transpose(1, 2)).sub_((da * a).sum(-1, keepdim=True)).mul_(p)
            s["dv"][k0:k0 + lk] = (p.transpose(1, 2) @ da).transpose(0, 1)
            s["dq"][q0:q0 + lq] = back((ds @ k) * scale)
            s["dk"][k0:k0 + lk] = ((ds.transpose(1, 2) @ q) * scale).transpose(0, 1)


SCALED = {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 4.0},
          "parts": {"factor": 8.0, "original_positions": 4096, "slow": 1.0, "fast": 32.0}}


def _frequencies(c):
    """Turning of each pair by a position (radians, 64 bits), and the amplitude."""
    n, how = c["rotary_dim"], SCALED[c["scaling"]]
    i = torch.arange(n // 2, device="cuda", dtype=torch.float64)
    base = BASE * how["factor"] ** (n / (n - 2)) if c["scaling"] == "base" and n > 2 else BASE
    f = base ** (-2.0 * i / n)
    if c["scaling"] == "linear":
        return f / how["factor"], 1.0
    if c["scaling"] == "parts":   # few turns in the original context: stretched; many: left as they are
        turns = how["original_positions"] * f / (2 * math.pi)
        keep = ((turns - how["slow"]) / (how["fast"] - how["slow"])).clamp(0, 1)
        return f * keep + f / how["factor"] * (1 - keep), 0.1 * math.log(how["factor"]) + 1.0
    return f, 1.0


def _turned(c, x, cos, sin):
    n = c["rotary_dim"]
    x = x.to(cos.dtype)
    if c["layout"] == "half":
        u, w = x[..., :n // 2], x[..., n // 2:n]
        return torch.cat([u * cos - w * sin, u * sin + w * cos, x[..., n:]], -1)
    u, w = x[..., 0:n:2], x[..., 1:n:2]
    return torch.cat([torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2), x[..., n:]], -1)


def _plain_rotary(c, s):
    f, amplitude = _frequencies(c)
    angle = (s["positions"].double()[:, None] * f)[:, None]
    cos, sin = ((t * amplitude).float() for t in (angle.cos(), angle.sin()))
    s["q_out"].copy_(_turned(c, s["q"], cos[:, :, None], sin[:, :, None]))
    s["k_out"].copy_(_turned(c, s["k"], cos, sin))
    s["dq"].copy_(_turned(c, s["dq_out"], cos[:, :, None], -sin[:, :, None]))
    s["dk"].copy_(_turned(c, s["dk_out"], cos, -sin))


def _grouped(c, x):
    """The columns that share a scale in a dimension of their own, zeros behind the last."""
    n = c["columns"] or c["hidden"]
    pad = -c["hidden"] % n
    return torch.nn.functional.pad(x, (0, pad)).view(c["tokens"], -1, n)


def _plain_rmsnorm(c, s):
    h = c["hidden"]
    s["xsum"].copy_(s["x"].float() + s["residual"].float())
    x, gamma = s["xsum"].float(), s["gamma"].float()   # the sum as it is stored is what is normalised
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    s["rstd"].copy_(rstd[:, 0])
    if c["eight_bits"]:
        y = _grouped(c, x * rstd * gamma)
        most = y.abs().amax(-1, keepdim=True)
        scale = torch.where(most > 0, most / E4M3_MOST, 1.0)
        s["scale"].copy_(scale[..., 0])
        s["out"].copy_((y / scale).clamp(-E4M3_MOST, E4M3_MOST).view(c["tokens"], -1)[:, :h].to(torch.float8_e4m3fn))
        return
    s["out"].copy_(x * rstd * gamma)
    if c["backward"]:
        dout = s["dout"].float()
        dn = dout * gamma
        xn = x * rstd
        s["dx"].copy_(s["dres"].float() + rstd * (dn - xn * (dn * xn).mean(-1, keepdim=True)))
        s["dgamma"].copy_((dout * xn).sum(0))


# ------------------------------------------------------------------ one pass
def _own_attention(c, s):
    import paper_2201_11990_amd as M
    where = (s["q_offsets"], s["k_offsets"], s["max_q"], s["max_k"])
    if "workspace" not in s:   # kept from step to step, as a training program or a server does
        desc = M.packed_desc(s["q"], s["k"], len(s["q_offsets"]) - 1, s["max_q"], s["max_k"])
        size = M.mtnlg_packed_attention_bwd_workspace(desc) if c["backward"] else 0
        s["workspace"] = torch.empty(max(size, M.mtnlg_packed_attention_fwd_workspace(desc)), dtype=torch.uint8, device="cuda")
    M.mtnlg_packed_attention_fwd(s["q"], s["k"], s["v"], s["a"], s["lse"], *where, k_lengths=s["k_lengths"], workspace=s["workspace"])
    if c["backward"]:
        M.mtnlg_packed_attention_bwd(s["q"], s["k"], s["v"], s["a"], s["lse"], s["da"], s["dq"], s["dk"], s["dv"], *where,
                                     k_lengths=s["k_lengths"], workspace=s["workspace"])


def _own_rotary(c, s):
    import paper_2201_11990_amd as M
    desc = M.rotary_desc(c["rotary_dim"], layout=M.ROTARY_HALF if c["layout"] == "half" else M.ROTARY_INTERLEAVED, base=BASE,
                         scaling={"none": M.ROTARY_UNSCALED, "linear": M.ROTARY_LINEAR, "base": M.ROTARY_BASE, "parts": M.ROTARY_PARTS}[c["scaling"]],
                         **SCALED[c["scaling"]])
    M.mtnlg_rotary_fwd(desc, s["q"], s["k"], s["q_out"], s["k_out"], positions=s["positions"])
    M.mtnlg_rotary_bwd(desc, s["dq_out"], s["dk_out"], s["dq"], s["dk"], positions=s["positions"])


def _own_rmsnorm(c, s):
    import paper_2201_11990_amd as M
    if c["eight_bits"]:
        M.mtnlg_rmsnorm_fwd_e4m3(s["x"], s["gamma"], EPS, s["out"], s["scale"], s["rstd"], columns=c["columns"], residual=s["residual"],
                                 xsum=s["xsum"])
        return
    M.mtnlg_rmsnorm_fwd(s["x"], s["gamma"], EPS, s["out"], s["rstd"], residual=s["residual"], xsum=s["xsum"])
    if c["backward"]:
        if "workspace" not in s:
            s["workspace"] = torch.empty(M.mtnlg_rmsnorm_bwd_workspace(c["tokens"], c["hidden"]), dtype=torch.uint8, device="cuda")
        M.mtnlg_rmsnorm_bwd(s["xsum"], s["gamma"], s["rstd"], s["dout"], s["dx"], s["dgamma"], s["workspace"], dres=s["dres"])


def _results(c):
    if c["kind"] == "attention":
        return ("a", "lse", "dq", "dk", "dv") if c["backward"] else ("a", "lse")
    if c["kind"] == "rotary":
        return ("q_out", "k_out", "dq", "dk")
    if c["eight_bits"]:
        return ("xsum", "out", "scale", "rstd")
    return ("xsum", "out", "rstd", "dx", "dgamma") if c["backward"] else ("xsum", "out", "rstd")


def run(state):
    c = state["case"]
    if own:
        {"attention": _own_attention, "rotary": _own_rotary, "rmsnorm": _own_rmsnorm}[c["kind"]](c, state)
    else:
        {"attention": _plain_attention, "rotary": _plain_rotary, "rmsnorm": _plain_rmsnorm}[c["kind"]](c, state)
    return {k: state[k] for k in _results(c)}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "attention":
        ql, kl = _lengths(c["queries"]), _lengths(c["keys"])
        kv, heads, d = c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"]
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(ql, kl))   # of queries and keys that they see
        rows, keys = sum(ql) * heads, sum(kl) * kv
        # forward: q, k, v in, a and lse out, two products of d each; backward: those and da in, dq, dk, dv out, five products
        forward = es * d * (2 * rows + 2 * keys) + 4 * rows
        return {"bytes": forward + (es * d * (4 * rows + 4 * keys) + 4 * rows if c["backward"] else 0),
                "flops": (7.0 if c["backward"] else 2.0) * 2.0 * d * pairs * heads}
    if c["kind"] == "rotary":   # forward and backward each read and write queries and keys
        n = c["tokens"] * c["kv_heads"] * (c["group"] + 1) * c["head_dim"]
        return {"bytes": 4 * n * es + 8 * c["tokens"], "flops": 6.0 * n}
    t, h = c["tokens"], c["hidden"]
    if c["eight_bits"]:   # x and residual in, their sum, the codes and their scales out
        return {"bytes": t * h * (3 * es + 1) + 4 * t * (1 + -(-h // (c["columns"] or h))) + h * es, "flops": 8.0 * t * h}
    # forward: x and residual in, sum and result out; backward: sum, dout, dres in, dx out
    return {"bytes": t * h * es * (8 if c["backward"] else 4) + 4 * t + h * (es + 4), "flops": (16.0 if c["backward"] else 5.0) * t * h}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_attention(c, s):
    ql, kl, q_off, k_off = s["host"]
    kv, r, d = c["kv_heads"], c["group"], c["head_dim"]
    out = {k: torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in _results(c)}
    for n in range(len(ql)):
        lq, lk = ql[n], kl[n]
        if lq == 0:
            continue
        qs, ks = slice(q_off[n], q_off[n] + lq), slice(k_off[n], k_off[n] + lk)
        seen = torch.ones(lq, lk, dtype=torch.bool, device="cuda").tril(lk - lq)
        for j in range(kv):
            k, v = s["k"][ks, j].double(), s["v"][ks, j].double()
            for i in range(r):
                q = s["q"][qs, j, i].double()
                sc = torch.where(seen, (q @ k.T) / math.sqrt(d), -math.inf)
                lse = torch.logsumexp(sc, -1, keepdim=True)
                p = torch.exp(sc - lse)
                out["a"][qs, j, i] = p @ v
                out["lse"][j * r + i, qs] = lse[:, 0]
                if c["backward"]:
                    da = s["da"][qs, j, i].double()
                    dp = da @ v.T
                    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(d)
                    out["dq"][qs, j, i] = ds @ k
                    out["dk"][ks, j] += ds.T @ q
                    out["dv"][ks, j] += p.T @ da
    return out


def _exact_rotary(c, s):
    f, amplitude = _frequencies(c)
    n = c["rotary_dim"]
    turn = torch.polar(torch.full((c["tokens"], n // 2), amplitude, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * f)

    def turned(x, by):
        x = x.double()
        pairs = torch.stack([x[..., :n // 2], x[..., n // 2:n]], -1) if c["layout"] == "half" else x[..., :n].unflatten(-1, (n // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by.view(c["tokens"], *[1] * (x.dim() - 2), n // 2))
        z = torch.cat([z[..., 0], z[..., 1]], -1) if c["layout"] == "half" else z.flatten(-2)
        return torch.cat([z, x[..., n:]], -1)

    return {"q_out": turned(s["q"], turn), "k_out": turned(s["k"], turn), "dq": turned(s["dq_out"], turn.conj()), "dk": turned(s["dk_out"], turn.conj())}


def _exact_rmsnorm(c, s):
    total = s["x"].double() + s["residual"].double()
    x = total.to(DTYPES[c["dtype"]]).double().requires_grad_()
    gamma = s["gamma"].double().requires_grad_()
    rstd = torch.rsqrt(x.square().mean(-1) + EPS)
    y = x * rstd[:, None] * gamma
    out = {"xsum": total, "rstd": rstd.detach()}
    if c["eight_bits"]:
        y = y.detach()
        parts = y.split(c["columns"] or c["hidden"], -1)
        out["scale"] = torch.stack([p.abs().amax(-1) for p in parts], -1) / E4M3_MOST
        out["out"] = torch.cat([p / out["scale"][:, i:i + 1] for i, p in enumerate(parts)], -1).float().to(torch.float8_e4m3fn).double()
        return out
    if c["backward"]:
        y.backward(s["dout"].double())
        out.update(dx=x.grad + s["dres"].double(), dgamma=gamma.grad)
    return {**out, "out": y.detach()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "rotary": _exact_rotary, "rmsnorm": _exact_rmsnorm}[case["kind"]](case, s)
