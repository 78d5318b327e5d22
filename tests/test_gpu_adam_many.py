"""AdamW over many tensors at once and the squared norm of their gradients, against 64 bits.

f = 2^-23 for every operation in fp32.  A moment is off by 3 f (|old part| + |new part|); its code may differ from that of the 64-bit moment only where
quotient / step + u lies as near to a whole number as the quotient's error: that of the moment over the scale, and 8 f of the quotient for the
scale, its reciprocal, the product and the root; 2^-20 more below 2^-6, where 2^-6 is added first."""
import math

import pytest
import torch

import paper_2201_11990_amd as M

pytestmark = pytest.mark.gpu
F, BLOCK = 2.0 ** -23, 256
COUNTS = {"one": [1], "small": [1, 3, 255, 256, 257, 520, 4, 4095, 4096, 4097], "mixed": [70_001, 2, 12_288, 1_000_003, 511],
          "many": [(37 * i * i) % 4999 + 1 for i in range(200)]}
E4M3 = torch.float8_e4m3fn


def model(counts, grads, seed=0, scale=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(counts):
        r = lambda f: torch.randn(n, generator=g, device="cuda") * f   # noqa: E731
        out.append({"master": r(0.02), "grad": (r(scale) * torch.exp(r(1.0))).to(torch.bfloat16 if grads == "bf16" else torch.float32),
                    "weight_bf16": torch.full((n,), float("nan"), dtype=torch.bfloat16, device="cuda") if i % 3 != 2 else None, "decay": i % 2 == 0})
    return out


def with_states(rows, bits, seed=1, zero=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in rows:
        n = t["master"].numel()
        if bits == 32:
            t["m"] = torch.zeros(n, device="cuda") if zero else torch.randn(n, generator=g, device="cuda") * 1e-3
            t["v"] = torch.zeros(n, device="cuda") if zero else torch.randn(n, generator=g, device="cuda").square() * 1e-6
        else:
            b = -(-n // BLOCK)
            codes = lambda lo: torch.randint(lo, 127, (n,), generator=g, device="cuda", dtype=torch.uint8)   # noqa: E731
            sign = torch.randint(0, 2, (n,), generator=g, device="cuda", dtype=torch.uint8) * 128
            t["m"] = (torch.zeros(n, dtype=torch.uint8, device="cuda") if zero else codes(0) + sign).view(E4M3)
            t["v"] = (torch.zeros(n, dtype=torch.uint8, device="cuda") if zero else codes(1)).view(E4M3)
            for k in ("m_scale", "v_scale"):
                t[k] = torch.zeros(b, device="cuda") if zero else (0.5 + torch.rand(b, generator=g, device="cuda")) * 1e-5
    return rows


def spread(scale, n):
    return scale.double().repeat_interleave(BLOCK)[:n]


def copies(rows):
    return [{k: (v.clone() if isinstance(v, torch.Tensor) else v) for k, v in t.items()} for t in rows]


LOW, WHOLE = 0xFFFFFFFF, (1 << 64) - 1


def numbers(seed, step, first_block, n):
    """u of m and of the root for each element of a tensor whose blocks begin at first_block"""
    s = (seed * 0x9E3779B97F4A7C15 + step) & WHOLE
    for shift, by in ((32, 0xBB67AE8584CAA73B), (29, 0x6A09E667F3BCC909)):
        s = ((s ^ (s >> shift)) * by) & WHOLE
    s ^= s >> 32
    i = torch.arange(n, device="cuda")
    wrap = lambda x, by: (x * by) & LOW   # noqa: E731
    k = (wrap(first_block + i // BLOCK, 0x9E3779B1) + (s & LOW)) & LOW
    k = wrap(k ^ (k >> 15), 0x510E527F)
    k = k ^ (k >> 13) ^ (s >> 32)
    h = (k + wrap(i % BLOCK, 0x3C6EF373)) & LOW
    h = wrap(h ^ (h >> 16), 0x6A09E667)
    h = wrap(h ^ (h >> 15), 0xBB67AE85)
    h = h ^ (h >> 16)
    return ((h & 0xFFFF).double() + 0.5) / 65536, ((h >> 16).double() + 0.5) / 65536


def codes_of(x, error, u, least):
    """Codes as values, scales, and where a code may be another one"""
    n = x.numel()
    most = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK)).view(-1, BLOCK).amax(1)
    scale = torch.where(most > 0, (most / 448).clamp(min=2.0 ** -126), 1.0)
    wide = spread(scale, n)
    y = (x.abs() / wide).clamp(max=448)
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    t = y / step + u
    # of the smaller step below: a quotient on the other side of a power of two is counted in steps of half the size, and 8 steps from there on are 16 below
    near = (t - t.round()).abs() <= (error / wide + 8 * F * y) / (step / 2) + 2.0 ** -20
    k = torch.floor(t)
    return torch.sign(x) * torch.where(x != 0, k.clamp(min=least), 0.0) * step, scale, near


def check(before, after, bits, norm, step, seed=0, lr=1e-3, clip=1.0, b1=0.9, b2=0.95, eps=1e-8, wd=0.1, block=0):
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))   # noqa: E731
    b1, b2, lr, wd, eps = map(f32, (b1, b2, lr, wd, eps))
    coef = min(1.0, clip / (math.sqrt(norm) + 1e-6)) if norm is not None and clip > 0 else 1.0
    for old, new in zip(before, after):
        n = old["master"].numel()
        p, g = old["master"].double(), old["grad"].double() * coef
        m, v = old["m"].double() if bits == 32 else old["m"].float().double() * spread(old["m_scale"], n), None
        v = old["v"].double() if bits == 32 else (old["v"].float().double() * spread(old["v_scale"], n)) ** 2
        em, ev = 3 * F * (b1 * m.abs() + (1 - b1) * g.abs()), 4 * F * (b2 * v + (1 - b2) * g * g)
        if coef != 1.0:   # the norm rounds to fp32, its root and the quotient once each: 3 f more of the gradients
            em, ev = em + 3 * F * (1 - b1) * g.abs(), ev + 6 * F * (1 - b2) * g * g
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        mh, vh = m / (1 - b1 ** step), v / (1 - b2 ** step)
        update = mh / (vh.sqrt() + eps) + (wd * p if old.get("decay", True) else 0)
        want = p - lr * update
        # v is off by ev / v relative, half of that in its root; five more operations
        error = lr * ((em / (1 - b1 ** step) + mh.abs() * (0.5 * ev / v.clamp(min=1e-300) + 8 * F)) / (vh.sqrt() + eps) + 4 * F * update.abs()) + F * want.abs()
        ok = lambda got, value, bound, what: (((got.double() - value).abs() <= bound).all() or pytest.fail(f"{what}: {float(((got.double() - value).abs() - bound).max())}"))   # noqa: E731
        ok(new["master"], want, error, "weight")
        if old.get("weight_bf16") is not None:
            assert torch.equal(new["weight_bf16"], new["master"].bfloat16())
        assert torch.equal(new["grad"].view(torch.uint8), old["grad"].view(torch.uint8))
        if bits == 32:
            ok(new["m"], m, em + 2.0 ** -149, "m")
            ok(new["v"], v, ev + 2.0 ** -148, "v")
        else:
            um, uv = numbers(seed, step, block, n)
            root = v.sqrt()
            for k, x, e, u, least in (("m", m, em, um, 0), ("v", root, 0.5 * ev / root.clamp(min=1e-300) + F * root, uv, 1)):
                codes, scale, near = codes_of(x, e, u, least)
                ok(new[k + "_scale"], scale, scale * (4 * F) + (e.max() / 448), k + " scale")
                got = new[k].float().double()
                same = got == codes
                assert (same | near).all(), (k, int((~(same | near)).sum()))
                assert near.double().mean() < 1e-2 + 2 / n
                # what differs is the neighbouring code
                wide = torch.maximum(got.abs(), codes.abs()).clamp(min=2.0 ** -6)
                assert ((got - codes).abs() <= 2.0 ** -3 * wide + 2.0 ** -9).all()
        block += -(-n // BLOCK)


def norm_of(rows):
    return sum(float(t["grad"].double().square().sum()) for t in rows)


def run_norm(table, fill=float("nan")):
    sq = torch.full((1,), fill, device="cuda")
    ws = torch.full((M.mtnlg_grad_sqnorm_many_workspace(),), 0xFF, dtype=torch.uint8, device="cuda")
    M.mtnlg_grad_sqnorm_many(table, sq, ws)
    return sq, ws


@pytest.mark.parametrize("grads", ["fp32", "bf16"])
@pytest.mark.parametrize("which", list(COUNTS))
def test_norm(grads, which):
    rows = model(COUNTS[which], grads)
    sq, ws = run_norm(rows)
    want = norm_of(rows)
    assert abs(float(sq) - want) <= 2.0 ** -24 * want * 1.01   # 64-bit sums, one rounding
    again = torch.full((1,), 3.0, device="cuda")
    M.mtnlg_grad_sqnorm_many(rows, again, ws, accumulate=True)
    assert abs(float(again) - (3.0 + want)) <= 2.0 ** -24 * (3.0 + want) * 1.01
    both, _ = run_norm(M.AdamTensors([{"grad": t["grad"]} for t in rows]))
    assert torch.equal(both, sq)


@pytest.mark.parametrize("grads", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("which", list(COUNTS))
def test_three_steps(bits, grads, which):
    rows = with_states(model(COUNTS[which], grads), bits)
    table = M.AdamTensors(rows)
    assert len(table) == len(rows)
    for step, clip in ((1, 0.0), (2, 1e-3), (700, 1.0)):
        before = copies(rows)
        sq, _ = run_norm(table)
        M.mtnlg_adam_step_many(table, sq, lr=1e-3, step=step, max_grad_norm=clip, seed=step * 77)
        check(before, rows, bits, float(sq), step, seed=step * 77, clip=clip)


@pytest.mark.parametrize("grads", ["fp32", "bf16"])
@pytest.mark.parametrize("clip", [0.0, 1e-2])
def test_codes_and_scales_bit_by_bit(grads, clip):
    # every operation rounds once to fp32, here as there
    rows = with_states(model(COUNTS["small"] + [50_001, 4096 * 3], grads, 3), 8, 4)
    before = [{k: (v.cpu() if isinstance(v, torch.Tensor) else v) for k, v in t.items()} for t in rows]
    sq, _ = run_norm(rows)
    M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=12, max_grad_norm=clip, seed=987654321987654321)
    f = torch.tensor([0.9, 0.95, 1e-6, clip], dtype=torch.float32)
    b1, b2, one = f[0], f[1], torch.ones((), dtype=torch.float32)
    root = lambda x: x.double().sqrt().float()   # noqa: E731  (of 53 bits to 24: the same as rounding once)
    coef = torch.minimum(one, f[3] / (root(sq.cpu()) + f[2])) if clip > 0 else one
    block = 0
    for old, new in zip(before, rows):
        n = old["master"].numel()
        wide = lambda s: s.repeat_interleave(BLOCK)[:n]   # noqa: E731
        g = old["grad"].float() * coef
        m = (old["m"].float() * wide(old["m_scale"])) * b1 + g * (one - b1)
        r = old["v"].float() * wide(old["v_scale"])
        r = root((r * r) * b2 + (g * (one - b2)) * g)
        for k, x, u, least in zip("mv", (m, r), numbers(987654321987654321, 12, block, n), (0, 1)):
            most = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK)).view(-1, BLOCK).amax(1)
            scale = torch.where(most > 0, (most * (one / 448)).clamp(min=2.0 ** -126), one)
            assert torch.equal(new[k + "_scale"].cpu(), scale), k
            y = (x.abs() * wide(one / scale)).clamp(max=448).double()
            step = torch.exp2((torch.frexp(y).exponent - 1).clamp(min=-6).double() - 3)
            steps = torch.floor(y / step + u.cpu())
            codes = torch.copysign(torch.where(x != 0, steps.clamp(min=least), 0.0) * step, x.double()).float().to(E4M3)
            assert torch.equal(new[k].cpu().view(torch.uint8), codes.view(torch.uint8)), k
        block += -(-n // BLOCK)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_nothing_and_without_a_norm(bits):
    rows = with_states(model(COUNTS["small"], "fp32"), bits, zero=True)
    before = copies(rows)
    M.mtnlg_adam_step_many(rows, lr=1e-3, step=1, seed=5)
    check(before, rows, bits, None, 1, seed=5)


@pytest.mark.parametrize("bits", [32, 8])
def test_nothing_comes_of_nothing_whatever_eps(bits):
    rows = with_states(model([1000], "fp32"), bits, zero=True)
    rows[0]["grad"].zero_()
    before = copies(rows)
    M.mtnlg_adam_step_many(rows, lr=1e-3, step=1, eps=1e-42, weight_decay=0.0)
    for k in ("master", "m", "v"):
        assert torch.equal(rows[0][k].view(torch.uint8), before[0][k].view(torch.uint8)), k


@pytest.mark.parametrize("bits", [32, 8])
def test_a_gradient_that_two_tensors_share(bits):
    rows = with_states(model([5000, 5000, 300], "bf16"), bits)
    rows[1]["grad"] = rows[0]["grad"]
    before = copies(rows)
    sq, _ = run_norm(rows)
    want = norm_of(rows)
    assert abs(float(sq) - want) <= 2.0 ** -24 * want * 1.01
    M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=2, seed=9)
    check(before, rows, bits, float(sq), 2, seed=9)


def test_many_launches_of_small_tensors():
    # 1500 tensors side by side in one buffer: 27 launches, and norms of 10
    sizes = [(i * 37) % 61 * 4 + 4 for i in range(1500)]
    flat = with_states(model([sum(sizes)], "fp32"), 32)[0]
    one = copies([flat])[0]
    rows, at = [], 0
    for n in sizes:
        rows.append({k: (v[at:at + n] if isinstance(v, torch.Tensor) else v) for k, v in flat.items()})
        at += n
    sq, _ = run_norm(rows)
    want = norm_of([flat])
    assert abs(float(sq) - want) <= 2.0 ** -24 * want * 1.01
    M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=3)
    M.mtnlg_adam_step_many([one], sq, lr=1e-3, step=3)
    for k in ("master", "m", "v", "weight_bf16"):
        assert torch.equal(flat[k], one[k]), k


def test_states_of_32_bits_as_the_step_on_one_tensor():
    rows = with_states(model(COUNTS["mixed"], "fp32"), 32)
    one = copies(rows)
    sq = torch.full((1,), norm_of(rows), device="cuda")
    M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=3)
    for t, w in zip(rows, one):
        M.mtnlg_adam_step(w["master"], w["m"], w["v"], w["grad"], w["weight_bf16"], sq, lr=1e-3, step=3, weight_decay=0.1 if w["decay"] else 0.0)
        for k in ("master", "m", "v"):   # both within a few f of the same value
            assert (t[k] - w[k]).abs().max() <= 8 * F * w[k].abs().max()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_a_norm_that_is_not_finite_leaves_all_as_it_was(bits, bad):
    rows = with_states(model(COUNTS["small"], "bf16"), bits)
    rows[3]["grad"][7] = bad
    before = copies(rows)
    sq, _ = run_norm(rows)
    assert not math.isfinite(float(sq))
    for clip in (1.0, 0.0):
        M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=3, max_grad_norm=clip)
    for t, w in zip(rows, before):
        assert all(torch.equal(t[k].view(torch.uint8), w[k].view(torch.uint8)) for k in t if isinstance(t[k], torch.Tensor))


def test_nan_and_infinities_without_a_norm_stay_in_their_block():
    rows = with_states(model([1000], "fp32"), 8)
    clean = copies(rows)
    rows[0]["grad"][300] = float("nan")
    M.mtnlg_adam_step_many(clean, lr=1e-3, step=3)
    M.mtnlg_adam_step_many(rows, lr=1e-3, step=3)
    t, w = rows[0], clean[0]
    assert torch.isnan(t["master"][300]) and torch.isnan(t["m"][300].float()) and torch.isnan(t["v"][300].float())
    other = torch.arange(1000, device="cuda") // BLOCK != 1
    same = torch.arange(1000, device="cuda") != 300
    assert torch.equal(t["master"][same], w["master"][same])
    for k in ("m", "v"):
        assert torch.equal(t[k].view(torch.uint8)[other], w[k].view(torch.uint8)[other]) and torch.isfinite(t[k + "_scale"]).all()


def test_codes_round_without_bias_and_slow_moments_move():
    # every block holds one element of 448 and others of one value between two codes: 1.7 of a step from one to the next is rounded up in 70 % of them
    n = BLOCK * 4096
    grad = torch.full((n,), 9.7 / 448, device="cuda")
    grad[::BLOCK] = 1.0
    row = with_states([{"master": torch.zeros(n, device="cuda"), "grad": grad}], 8, zero=True)[0]
    M.mtnlg_adam_step_many([row], lr=0.0, step=1, beta1=0.0, beta2=0.0, seed=11)
    rest = torch.arange(n, device="cuda") % BLOCK != 0
    for k in ("m", "v"):
        codes = row[k].float()[rest]
        assert ((codes == 9) | (codes == 10)).all()
        share = float((codes == 10).double().mean())
        assert abs(share - 0.7) <= 5 * math.sqrt(0.21 / codes.numel()), (k, share)   # five standard deviations
    one = row["m"].clone()
    joint = ((row["m"].float()[rest] == 10) & (row["v"].float()[rest] == 10)).double().mean()   # of the two moments independently
    assert abs(float(joint) - 0.49) <= 5 * math.sqrt(0.25 / int(rest.sum()))
    neighbours = (row["m"].float().view(-1, BLOCK)[:, 1:-1] == 10) & (row["m"].float().view(-1, BLOCK)[:, 2:] == 10)
    assert abs(float(neighbours.double().mean()) - 0.49) <= 5 * math.sqrt(0.25 / neighbours.numel() * 3)   # (pairs overlap: three times the variance at most)
    for kw in (dict(seed=12), dict(seed=11, step=2)):
        M.mtnlg_adam_step_many([row], lr=0.0, **{"step": 1, "beta1": 0.0, "beta2": 0.0, **kw})
        assert not torch.equal(one.view(torch.uint8), row["m"].view(torch.uint8))
    # an average of a constant: beta2 = 0.999 takes a thousandth of what is left a step, a tenth of a code's step and less
    row = with_states([{"master": torch.zeros(n, device="cuda"), "grad": torch.ones(n, device="cuda")}], 8, zero=True)[0]
    row["grad"][::2] = 0.25
    table = M.AdamTensors([row])
    for step in range(1, 201):
        M.mtnlg_adam_step_many(table, lr=0.0, step=step, beta2=0.999, seed=3)
    v = (row["v"].float().view(-1, BLOCK) * row["v_scale"][:, None]).view(-1).double()
    exact = 1 - 0.999 ** 200
    # rounding adds at most a variance of (step / 2)^2 of the root a step: means of squares are too large by the spread alone, 200 steps of (2^-4)^2 / 4 at the most
    for part, want in ((v[1::2], exact), (v[::2], exact / 16)):
        mean = float(part.square().mean() / want)
        assert 0.97 <= mean <= 1 + 200 * 2.0 ** -10, mean


@pytest.mark.parametrize("bits", [32, 8])
def test_runs_are_identical_and_replays_too(bits):
    start = with_states(model(COUNTS["mixed"] + COUNTS["many"], "bf16"), bits)
    rows = copies(start)
    table = M.AdamTensors(rows)
    sq, ws = run_norm(table)

    def put():
        for t, w in zip(rows, start):
            for k in t:
                if isinstance(t[k], torch.Tensor):
                    t[k].copy_(w[k])

    def run():
        M.mtnlg_grad_sqnorm_many(table, sq, ws)
        M.mtnlg_adam_step_many(table, sq, lr=1e-3, step=9, seed=4)

    run()
    want = copies(rows)
    same = lambda: all(torch.equal(t[k].view(torch.uint8), w[k].view(torch.uint8)) for t, w in zip(rows, want) for k in t if isinstance(t[k], torch.Tensor))   # noqa: E731
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        put()
        sq.fill_(float("nan")), ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert same()
    put()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    assert same()


@pytest.mark.parametrize("bits,grads", [(32, "fp32"), (8, "bf16")])
def test_a_tensor_of_more_than_32_bits_of_elements(bits, grads):
    n = (1 << 31) + 4096 * 3 + 77
    gdt = torch.bfloat16 if grads == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(5)
    part = torch.randn(1 << 20, generator=g, device="cuda") * 1e-3
    whole = lambda x, dt: x.to(dt).repeat(-(-n // x.numel()))[:n].contiguous()   # noqa: E731
    row = {"master": whole(part * 20, torch.float32), "grad": whole(part, gdt), "weight_bf16": torch.empty(n, dtype=torch.bfloat16, device="cuda")}
    if bits == 32:
        row.update(m=whole(part * 0.5, torch.float32), v=whole(part.square(), torch.float32))
    else:
        codes = torch.randint(1, 127, (1 << 20,), generator=g, device="cuda", dtype=torch.uint8)
        row.update(m=whole(codes, torch.uint8).view(E4M3), v=whole(codes.flip(0), torch.uint8).view(E4M3))
        row.update({k: torch.full((-(-n // BLOCK),), 1e-6, device="cuda") for k in ("m_scale", "v_scale")})
    other = with_states(model([700], grads, 9), bits)[0]
    rows = [other, row]
    want = norm_of([other]) + float(part.to(gdt).double().square().sum()) * (n // part.numel()) + float(part.to(gdt)[:n % part.numel()].double().square().sum())
    sq, _ = run_norm(rows)
    assert abs(float(sq) - want) <= 2.0 ** -24 * want * 1.01
    first = n // BLOCK - 40   # the last blocks, and some in between on either side of 2^31
    spans = [(first * BLOCK, n), ((1 << 31) - 2048, (1 << 31) + 2048), (0, 5000)]
    cut = lambda a, b: {k: (v if not isinstance(v, torch.Tensor) else v[a // BLOCK:-(-b // BLOCK)] if k.endswith("scale") else v[a:b]).clone()   # noqa: E731
                        if isinstance(v, torch.Tensor) else v for k, v in row.items()}
    before = [cut(a, b) for a, b in spans]
    M.mtnlg_adam_step_many(rows, sq, lr=1e-3, step=4, max_grad_norm=0.0, seed=6)
    for old, (a, b) in zip(before, spans):
        check([old], [cut(a, b)], bits, float(sq), 4, seed=6, clip=0.0, block=3 + a // BLOCK)
    del rows, row, before
    torch.cuda.empty_cache()


def test_what_lies_beside_the_tensors_is_left_as_it_was():
    for bits in (32, 8):
        for n in (1, 2, 3, 255, 257, 4099):
            whole, row = {}, with_states(model([n], "bf16"), bits)[0]
            for k in ("master", "m", "v", "weight_bf16", "m_scale", "v_scale"):
                if row.get(k) is not None:
                    whole[k] = torch.full(((row[k].numel() + 64) * row[k].element_size(),), 0x5A, dtype=torch.uint8, device="cuda")
                    part = whole[k][:row[k].numel() * row[k].element_size()].view(row[k].dtype)
                    row[k] = part.copy_(row[k])
            M.mtnlg_adam_step_many([row], lr=1e-3, step=1)
            assert all((w[row[k].numel() * row[k].element_size():] == 0x5A).all() for k, w in whole.items())


def test_training_a_gated_block_with_states_in_8_bits():
    """Forward, backward, norm and clipped step of the block on its weights, six times, beside the same in 64 bits with the library's own gradients."""
    T, h, ffn = 96, 264, 136
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s, f=1.0: torch.randn(s, generator=g, device="cuda") * f   # noqa: E731
    rows = []
    for shape, f in (((2 * ffn, h), h ** -0.5), ((h, ffn), ffn ** -0.5)):
        w = r(*shape, f=f)
        rows.append({"master": w, "weight_bf16": w.bfloat16(), "grad": torch.empty(shape, device="cuda")})
    w1, w2 = (t["weight_bf16"] for t in rows)
    with_states(rows, 8, zero=True)
    new = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    z, gg, y, dz, dx = new(T, 2 * ffn), new(T, ffn), new(T, h), new(T, 2 * ffn), new(T, h)
    x = r(T, h).bfloat16()
    desc = M.gated_desc(x, w1, M.GATE_SILU, flags=M.WGRAD_FP32)
    ws = torch.empty(max(16, M.mtnlg_gated_ffn_workspace(desc)), dtype=torch.uint8, device="cuda")
    table = M.AdamTensors(rows)
    for step in range(1, 7):
        before = copies(rows)
        dy = r(T, h).bfloat16()
        M.mtnlg_gated_ffn_fwd(desc, x, w1, w2, z, gg, y, ws)
        M.mtnlg_gated_ffn_bwd(desc, x, w1, w2, z, gg, dy, dz, dx, rows[0]["grad"], rows[1]["grad"], ws)
        for t, grad, a, b in ((rows[0], "dw_fc1", dz, x), (rows[1], "dw_fc2", dy, gg)):
            want, size = a.double().T @ b.double(), a.double().abs().T @ b.double().abs()
            assert ((t["grad"].double() - want).abs() <= F * (T + 2) * size).all(), grad
        for t, w in zip(before, rows):
            t["grad"] = w["grad"].clone()
        sq, _ = run_norm(table)
        M.mtnlg_adam_step_many(table, sq, lr=1e-3, step=step, seed=1)
        flat = lambda some: [{k: (v.flatten() if isinstance(v, torch.Tensor) else v) for k, v in t.items()} for t in some]   # noqa: E731
        check(flat(before), flat(rows), 8, float(sq), step, seed=1)
